// The calls a program makes most, marshalled natively: plain tensors on the current GPU and its current stream, outputs and
// workspace allocated here.  Every function returns None for anything else (another type, layout, device, a stream or a
// buffer of the caller's, a mode or transform of torch's that is active, a status that is not success); binding.py then
// takes its own path, which says what is wrong or does what this one does not.
//
// A call of a small problem is as long as its host side: hyena_se_fwd of 1 x 1024 x 256 fp32 took 6.9 us through ctypes, of
// which the checks, the output and the conversions were 3.3 and the launch 3; through here 4.1, where the kernel bounds it.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/VirtualGuardImpl.h>

#include "hyena.h"

namespace {

using Gated = decltype(&hyena_se_fwd);
using GatedBwd = decltype(&hyena_se_bwd);

// addresses in the loaded library (init), and torch's current raw stream by device index
struct Entries {
    Gated gated[2];
    GatedBwd bwd[2];
    decltype(&hyena_bwd_workspace_bytes) bwd_workspace;
    decltype(&hyena_chain_fwd) chain_fwd;
    decltype(&hyena_chain_workspace_bytes) chain_workspace;
    decltype(&hyena_chain_bwd) chain_bwd;
    decltype(&hyena_chain_bwd_workspace_bytes) chain_bwd_workspace;
    decltype(&hyena_li_fwd) li_fwd;
    decltype(&hyena_li_workspace_bytes) li_workspace;
    decltype(&hyena_rmsnorm_fwd) norm_fwd;
    decltype(&hyena_rmsnorm_bwd) norm_bwd;
    decltype(&hyena_rmsnorm_bwd_workspace_bytes) norm_bwd_workspace;
    decltype(&hyena_la_step) la_step;
    decltype(&hyena_sample) sample;
} e;
constexpr int kEntries = 16;
static_assert(sizeof(Entries) == kEntries * sizeof(void*), "a table of addresses");
PyObject* raw_stream = nullptr;

// Nothing that would have a say in the calls this file makes: torch function and dispatch modes, functorch transforms.
bool plain_context() {
    static const c10::DispatchKeySet usual({c10::DispatchKey::BackendSelect, c10::DispatchKey::ADInplaceOrView});
    return (c10::impl::tls_local_dispatch_key_set().included_ - usual).empty() && !at::impl::torch_function_mode_enabled();
}

const at::Tensor* plain(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    static const c10::DispatchKeySet wrapped({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                              c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                              c10::DispatchKey::Negative, c10::DispatchKey::ZeroTensor});
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.key_set().has_any(wrapped) || !t.is_contiguous())
        return nullptr;
    return &t;
}

// The type's code and the current stream of a tensor on the current GPU.
bool here(const at::Tensor& x, int& code, void*& stream) {
    const auto type = x.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) return false;
    if (c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice() != x.device()) return false;
    code = type == at::kFloat ? HY_F32 : HY_BF16;
    PyObject* index = PyLong_FromLong(x.device().index());
    if (!index) throw python_error();
    PyObject* s = PyObject_CallOneArg(raw_stream, index);
    Py_DECREF(index);
    if (!s) throw python_error();
    stream = PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (PyErr_Occurred()) throw python_error();
    return true;
}

struct Problem {
    int64_t B, L, D, group;
    int code;
    const at::Tensor* x[4];
    void* stream;
};

// n activations of one shape, on the current GPU
bool activations(PyObject* const* a, int n, PyObject* group, Problem& p) {
    if (!raw_stream || !plain_context() || !PyLong_CheckExact(group)) return false;
    for (int i = 0; i < n; ++i) {
        p.x[i] = plain(a[i]);
        if (!p.x[i]) return false;
    }
    const at::Tensor& x = *p.x[0];
    if (x.dim() != 3 || x.numel() == 0) return false;
    for (int i = 1; i < n; ++i)
        if (p.x[i]->sizes() != x.sizes() || p.x[i]->scalar_type() != x.scalar_type() || p.x[i]->device() != x.device()) return false;
    p.B = x.size(0);
    p.L = x.size(1);
    p.D = x.size(2);
    int overflow = 0;
    p.group = PyLong_AsLongLongAndOverflow(group, &overflow);
    if (overflow || p.group < 1 || p.group > 0x7fffffff) return false;
    return here(x, p.code, p.stream);
}

// taps per filter of a [D / group, taps] table beside the activations, or 0
int32_t filter(PyObject* o, const Problem& p, int64_t group, const at::Tensor*& t) {
    t = plain(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 2 || t->device() != p.x[0]->device() || p.D % group != 0 ||
        t->size(0) != p.D / group || t->size(1) < 1 || t->size(1) > 0x7fffffff)
        return 0;
    return (int32_t)t->size(1);
}

at::Tensor workspace(const Problem& p, int64_t bytes) {
    return bytes > 0 ? at::empty({bytes}, p.x[0]->options().dtype(at::kByte)) : at::Tensor();
}
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

template <typename F>
bool launched(F&& call) {
    hy_status rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc == HY_OK;
}

// (an undefined tensor is None)
PyObject* tuple_of(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) throw python_error();
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* o = THPVariable_Wrap(t);
        if (!o) {
            Py_DECREF(r);
            throw python_error();
        }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// (0: hyena_se_fwd, 1: hyena_mr_fwd; q, k, v, h, group)
PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Problem p;
    const at::Tensor* h;
    if (n != 6 || !activations(a + 1, 3, a[5], p)) Py_RETURN_NONE;
    const int32_t lh = filter(a[4], p, p.group, h);
    if (!lh) Py_RETURN_NONE;
    const Gated fn = e.gated[PyLong_AsLong(a[0]) != 0];
    at::Tensor y = at::empty_like(*p.x[0]);
    void *q = p.x[0]->data_ptr(), *k = p.x[1]->data_ptr(), *v = p.x[2]->data_ptr(), *out = y.data_ptr();
    const float* hp = static_cast<const float*>(h->data_ptr());
    if (!launched([&] { return fn(q, k, v, hp, out, p.B, p.L, p.D, lh, (int32_t)p.group, p.code, p.stream); })) Py_RETURN_NONE;
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// (0: hyena_se_bwd, 1: hyena_mr_bwd; dy, q, k, v, h, group)
PyObject* bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Problem p;
    const at::Tensor* h;
    if (n != 7 || !activations(a + 1, 4, a[6], p)) Py_RETURN_NONE;
    const int32_t lh = filter(a[5], p, p.group, h), group = (int32_t)p.group;
    if (!lh) Py_RETURN_NONE;
    const GatedBwd fn = e.bwd[PyLong_AsLong(a[0]) != 0];
    const int64_t need = e.bwd_workspace(p.B, p.L, p.D, lh, group, p.code);
    if (need < 0) Py_RETURN_NONE;
    const at::Tensor ws = workspace(p, need);
    const at::Tensor &dy = *p.x[0], dq = at::empty_like(dy), dk = at::empty_like(dy), dv = at::empty_like(dy), dh = at::empty_like(*h);
    void *yp = dy.data_ptr(), *q = p.x[1]->data_ptr(), *k = p.x[2]->data_ptr(), *v = p.x[3]->data_ptr(), *hp = h->data_ptr();
    void *o0 = dq.data_ptr(), *o1 = dk.data_ptr(), *o2 = dv.data_ptr(), *o3 = dh.data_ptr(), *wp = address(ws);
    if (!launched([&] {
            return fn(yp, q, k, v, static_cast<float*>(hp), o0, o1, o2, static_cast<float*>(o3), wp, need, p.B, p.L, p.D, lh, group,
                      p.code, p.stream);
        }))
        Py_RETURN_NONE;
    return tuple_of({dq, dk, dv, dh});
    END_HANDLE_TH_ERRORS
}

struct Chain {
    Problem p;
    const at::Tensor *f[3], *h;
    int32_t lf, lh, group, feat_group;
};
// n activations, hq, hk, hv, h, group, feat_group
bool chain(PyObject* const* a, int n, Chain& c) {
    if (!PyLong_CheckExact(a[n + 5]) || !activations(a, n, a[n + 4], c.p)) return false;
    int overflow = 0;
    const int64_t fg = PyLong_AsLongLongAndOverflow(a[n + 5], &overflow);
    if (overflow || fg < 1 || fg > 0x7fffffff) return false;
    c.feat_group = (int32_t)fg;
    c.group = (int32_t)c.p.group;
    c.lf = filter(a[n], c.p, fg, c.f[0]);
    if (!c.lf || filter(a[n + 1], c.p, fg, c.f[1]) != c.lf || filter(a[n + 2], c.p, fg, c.f[2]) != c.lf) return false;
    c.lh = filter(a[n + 3], c.p, c.group, c.h);
    return c.lh > 0;
}

// (q, k, v, hq, hk, hv, h, group, feat_group)
PyObject* chain_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Chain c;
    if (n != 9 || !chain(a, 3, c)) Py_RETURN_NONE;
    const Problem& p = c.p;
    const int64_t need = e.chain_workspace(p.B, p.L, p.D, c.lf, c.feat_group, c.lh, c.group, p.code);
    if (need < 0) Py_RETURN_NONE;
    const at::Tensor y = at::empty_like(*p.x[0]), ws = workspace(p, need);
    void* in[8];
    for (int i = 0; i < 3; ++i) {
        in[i] = p.x[i]->data_ptr();
        in[3 + i] = c.f[i]->data_ptr();
    }
    in[6] = c.h->data_ptr();
    in[7] = y.data_ptr();
    void* wp = address(ws);
    auto f = [&](int i) { return static_cast<const float*>(in[i]); };
    if (!launched([&] {
            return e.chain_fwd(in[0], in[1], in[2], f(3), f(4), f(5), f(6), in[7], wp, need, p.B, p.L, p.D, c.lf, c.feat_group,
                               c.lh, c.group, p.code, p.stream);
        }))
        Py_RETURN_NONE;
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// (dy, q, k, v, hq, hk, hv, h, group, feat_group)
PyObject* chain_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Chain c;
    if (n != 10 || !chain(a, 4, c)) Py_RETURN_NONE;
    const Problem& p = c.p;
    const int64_t need = e.chain_bwd_workspace(p.B, p.L, p.D, c.lf, c.feat_group, c.lh, c.group, p.code);
    if (need < 0) Py_RETURN_NONE;
    const at::Tensor ws = workspace(p, need);
    const at::Tensor dq = at::empty_like(*p.x[0]), dk = at::empty_like(*p.x[0]), dv = at::empty_like(*p.x[0]);
    const at::Tensor dhq = at::empty_like(*c.f[0]), dhk = at::empty_like(*c.f[1]), dhv = at::empty_like(*c.f[2]),
                     dh = at::empty_like(*c.h);
    void *in[8], *out[7] = {dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dhq.data_ptr(), dhk.data_ptr(), dhv.data_ptr(), dh.data_ptr()};
    for (int i = 0; i < 4; ++i) in[i] = p.x[i]->data_ptr();
    for (int i = 0; i < 3; ++i) in[4 + i] = c.f[i]->data_ptr();
    in[7] = c.h->data_ptr();
    void* wp = address(ws);
    auto f = [&](int i) { return static_cast<const float*>(in[i]); };
    auto g = [&](int i) { return static_cast<float*>(out[i]); };
    if (!launched([&] {
            return e.chain_bwd(in[0], in[1], in[2], in[3], f(4), f(5), f(6), f(7), out[0], out[1], out[2], g(3), g(4), g(5), g(6),
                               wp, need, p.B, p.L, p.D, c.lf, c.feat_group, c.lh, c.group, p.code, p.stream);
        }))
        Py_RETURN_NONE;
    return tuple_of({dq, dk, dv, dhq, dhk, dhv, dh});
    END_HANDLE_TH_ERRORS
}

// (q, k, v, R, lam, group)
PyObject* li(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Problem p;
    const at::Tensor *R, *lam;
    if (n != 6 || !activations(a, 3, a[5], p)) Py_RETURN_NONE;
    const int32_t order = filter(a[3], p, p.group, R), group = (int32_t)p.group;
    if (!order || filter(a[4], p, p.group, lam) != order) Py_RETURN_NONE;
    const int64_t need = e.li_workspace(p.B, p.L, p.D, order, group, p.code);
    if (need < 0) Py_RETURN_NONE;
    const at::Tensor y = at::empty_like(*p.x[0]), ws = workspace(p, need);
    void *q = p.x[0]->data_ptr(), *k = p.x[1]->data_ptr(), *v = p.x[2]->data_ptr(), *rp = R->data_ptr(), *lp = lam->data_ptr(),
         *out = y.data_ptr(), *wp = address(ws);
    if (!launched([&] {
            return e.li_fwd(q, k, v, static_cast<float*>(rp), static_cast<float*>(lp), out, wp, need, p.B, p.L, p.D, order, group,
                            p.code, p.stream);
        }))
        Py_RETURN_NONE;
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// None, or a plain tensor of these sizes and type on x's GPU; false for anything else
bool optional(PyObject* o, const at::Tensor& x, at::IntArrayRef sizes, at::ScalarType type, const at::Tensor*& t) {
    t = nullptr;
    if (o == Py_None) return true;
    t = plain(o);
    return t && t->sizes() == sizes && t->scalar_type() == type && t->device() == x.device();
}
void* address(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

// [..., D] activations of at least one row
const at::Tensor* rows(PyObject* o, int64_t& N, int64_t& D) {
    const at::Tensor* x = plain(o);
    if (!raw_stream || !plain_context() || !x || x->dim() < 1 || x->numel() == 0) return nullptr;
    D = x->size(-1);
    N = x->numel() / D;
    return x;
}

// (x, w, residual, eps, want_rstd, eight) -> (y, total, rstd), or with 8 bits (y, scale, total, rstd)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t N, D;
    int code;
    void* stream;
    const at::Tensor *x = n == 6 ? rows(a[0], N, D) : nullptr, *w, *r;
    if (!x || !PyFloat_CheckExact(a[3]) || !PyBool_Check(a[4]) || !PyBool_Check(a[5]) ||
        !optional(a[1], *x, x->sizes().slice(x->dim() - 1), x->scalar_type(), w) || !optional(a[2], *x, x->sizes(), x->scalar_type(), r) ||
        !here(*x, code, stream))
        Py_RETURN_NONE;
    const double eps = PyFloat_AS_DOUBLE(a[3]);
    const bool eight = a[5] == Py_True;
    auto of_rows = [&](bool wanted) { return wanted ? at::empty(x->sizes().slice(0, x->dim() - 1), x->options().dtype(at::kFloat)) : at::Tensor(); };
    const at::Tensor y = eight ? at::empty(x->sizes(), x->options().dtype(at::kFloat8_e4m3fn)) : at::empty_like(*x), scale = of_rows(eight),
                     total = r ? at::empty_like(*x) : at::Tensor(), rstd = of_rows(a[4] == Py_True);
    void *xp = x->data_ptr(), *rp = address(r), *wp = address(w), *yp = y.data_ptr(), *tp = address(total);
    float *const cp = static_cast<float*>(address(scale)), *const sp = static_cast<float*>(address(rstd));
    if (!launched([&] { return e.norm_fwd(xp, rp, wp, yp, cp, tp, sp, N, D, D, r ? D : 0, eps, code, stream); })) Py_RETURN_NONE;
    return eight ? tuple_of({y, scale, r ? total : *x, rstd}) : tuple_of({y, r ? total : *x, rstd});
    END_HANDLE_TH_ERRORS
}

// (dy, total, rstd, w, dtotal, want_dw) -> (dx, dw)
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    int64_t N, D;
    int code;
    void* stream;
    const at::Tensor *dy = n == 6 ? rows(a[0], N, D) : nullptr, *h, *s, *w, *dh;
    if (!dy || !PyBool_Check(a[5]) || !optional(a[1], *dy, dy->sizes(), dy->scalar_type(), h) || !h ||
        !optional(a[2], *dy, dy->sizes().slice(0, dy->dim() - 1), at::kFloat, s) || !s ||
        !optional(a[3], *dy, dy->sizes().slice(dy->dim() - 1), dy->scalar_type(), w) ||
        !optional(a[4], *dy, dy->sizes(), dy->scalar_type(), dh) || !here(*dy, code, stream))
        Py_RETURN_NONE;
    const bool want = w && a[5] == Py_True;
    const int64_t need = want ? e.norm_bwd_workspace(N, D, code) : 0;
    if (need < 0) Py_RETURN_NONE;
    const at::Tensor dx = at::empty_like(*dy), dw = want ? at::empty_like(*w) : at::Tensor(),
                     ws = need > 0 ? at::empty({need}, dy->options().dtype(at::kByte)) : at::Tensor();
    void *yp = dy->data_ptr(), *hp = h->data_ptr(), *sp = s->data_ptr(), *wp = address(w), *dhp = address(dh), *xp = dx.data_ptr(),
         *dwp = address(dw), *wsp = address(ws);
    if (!launched([&] { return e.norm_bwd(yp, hp, static_cast<float*>(sp), wp, dhp, xp, dwp, wsp, need, N, D, code, stream); })) Py_RETURN_NONE;
    return tuple_of({dx, dw});
    END_HANDLE_TH_ERRORS
}

// (q, k, v, g, state, scale) -> y
PyObject* la_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 6 || !raw_stream || !plain_context() || !PyFloat_CheckExact(a[5])) Py_RETURN_NONE;
    const at::Tensor* t[5];
    for (int i = 0; i < 5; ++i)
        if (!(t[i] = plain(a[i]))) Py_RETURN_NONE;
    const at::Tensor &q = *t[0], &k = *t[1], &v = *t[2], &g = *t[3], &state = *t[4];
    if (v.dim() != 3 || q.dim() != 3 || v.numel() == 0 || q.numel() == 0) Py_RETURN_NONE;
    const int64_t B = v.size(0), H = v.size(1), dv = v.size(2), dk = q.size(2), group = H / q.size(1);
    if (q.size(0) != B || H % q.size(1) != 0 || k.sizes() != q.sizes() || g.dim() != 2 || g.size(0) != B || g.size(1) != H ||
        state.dim() != 4 || state.size(0) != B || state.size(1) != H || state.size(2) != dk || state.size(3) != dv ||
        state.scalar_type() != at::kFloat || group > 0x7fffffff)
        Py_RETURN_NONE;
    for (int i = 0; i < 5; ++i)
        if (t[i]->device() != v.device() || (i < 4 && t[i]->scalar_type() != v.scalar_type())) Py_RETURN_NONE;
    int code;
    void* stream;
    if (!here(v, code, stream)) Py_RETURN_NONE;
    const double scale = PyFloat_AS_DOUBLE(a[5]);
    const at::Tensor y = at::empty_like(v);
    void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *gp = g.data_ptr(), *sp = state.data_ptr(), *yp = y.data_ptr();
    if (!launched([&] { return e.la_step(qp, kp, vp, gp, static_cast<float*>(sp), yp, B, H, (int32_t)group, dk, dv, scale, code, stream); }))
        Py_RETURN_NONE;
    return THPVariable_Wrap(y);
    END_HANDLE_TH_ERRORS
}

// A setting of every row, or the one number of all; false for anything else
bool setting(PyObject* o, const at::Tensor& x, at::IntArrayRef each, at::ScalarType type, double otherwise, const at::Tensor*& t, double& one) {
    one = otherwise;
    t = nullptr;
    if (o == Py_None) return true;
    if (PyFloat_CheckExact(o)) {
        one = PyFloat_AS_DOUBLE(o);
        return type == at::kFloat;
    }
    if (PyLong_CheckExact(o)) {
        int overflow = 0;
        const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
        one = (double)v;
        return !overflow && v > -(1 << 30) && v < 1 << 30;
    }
    return optional(o, x, each, type, t);
}

// (logits, u, temperature, top_k, top_p, min_p) -> (token, prob)
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor* z = n == 6 && raw_stream && plain_context() ? plain(a[0]) : nullptr;
    if (!z || z->dim() != 2 || z->numel() == 0) Py_RETURN_NONE;
    const int64_t N = z->size(0), V = z->size(1), each[1] = {N};
    const at::Tensor *u, *t, *k, *p, *m;
    double t1, k1, p1, m1;
    int code;
    void* stream;
    if (!optional(a[1], *z, each, at::kFloat, u) || !u || !setting(a[2], *z, each, at::kFloat, 1.0, t, t1) ||
        !setting(a[3], *z, each, at::kInt, 0.0, k, k1) || !setting(a[4], *z, each, at::kFloat, 1.0, p, p1) ||
        !setting(a[5], *z, each, at::kFloat, 0.0, m, m1) || !here(*z, code, stream))
        Py_RETURN_NONE;
    const at::Tensor token = at::empty(each, z->options().dtype(at::kLong)), prob = at::empty(each, z->options().dtype(at::kFloat));
    void *zp = z->data_ptr(), *up = u->data_ptr(), *tp = address(t), *kp = address(k), *pp = address(p), *mp = address(m), *op = token.data_ptr(),
         *qp = prob.data_ptr();
    auto f = [](void* x) { return static_cast<float*>(x); };
    if (!launched([&] {
            return e.sample(zp, f(up), f(tp), t1, static_cast<int32_t*>(kp), (int32_t)k1, f(pp), p1, f(mp), m1, static_cast<int64_t*>(op), f(qp), N, V,
                            N > 1 ? V : 0, code, stream);
        }))
        Py_RETURN_NONE;
    return tuple_of({token, prob});
    END_HANDLE_TH_ERRORS
}

// (addresses in the order of Entries, callable: device index -> raw stream)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 2 || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != kEntries || !PyCallable_Check(a[1])) {
        PyErr_SetString(PyExc_TypeError, "init(addresses, raw_stream)");
        return nullptr;
    }
    void* p[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], i));
        if (PyErr_Occurred()) return nullptr;
    }
    memcpy(&e, p, sizeof e);
    Py_INCREF(a[1]);
    Py_XSETREF(raw_stream, a[1]);
    Py_RETURN_NONE;
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(gated), FAST(bwd), FAST(chain_fwd), FAST(chain_bwd), FAST(li),
                         FAST(norm_fwd), FAST(norm_bwd), FAST(la_step), FAST(sample), FAST(init), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
