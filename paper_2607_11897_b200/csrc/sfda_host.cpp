// Native marshalling of the decode calls and of the operators of linear-attention layers: checks the tensors, takes their
// addresses and the current stream, calls the C ABI.  One token of one sequence keeps the GPU busy for 2.4 us; the same checks in
// Python with ctypes took 15 us.
// Errors as in the Python wrappers of the other calls: ValueError for layout and place, TypeError for the element type;
// what torch itself throws (a tensor without storage, no driver) comes back as the Python exception torch makes of it.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sfda.h"

namespace {

typedef int (*StepFn)(const void *, const void *, const void *, const float *, const float *, const float *, float *, void *, void *,
                      int, int, int, int, int, void *);
typedef int (*StepFusedFn)(const void *, const void *, const void *, const float *, const float *, const float *, float, float, float,
                           float, float *, void *, void *, int, int, int, int, int, void *);
StepFn g_step = nullptr;
StepFusedFn g_step_fused = nullptr;

// Address of a CUDA tensor of the wanted type; NULL for None where that is allowed.  false: a Python error is set.
bool address(PyObject *obj, const char *name, at::ScalarType type, void **out)
{
    *out = nullptr;
    if (obj == Py_None) return true;
    if (!THPVariable_Check(obj)) {
        PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
        return false;
    }
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s must be contiguous", name);
        return false;
    }
    if (!t.is_cuda()) {
        PyErr_Format(PyExc_ValueError, "%s must live on cuda", name);
        return false;
    }
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_TypeError, "%s must be %s", name, type == at::kFloat ? "torch.float32" : "torch.bfloat16");
        return false;
    }
    *out = t.data_ptr();
    return true;
}

bool stream_of(PyObject *obj, void **out)
{
    if (obj == Py_None) {
        *out = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject *h = PyObject_GetAttrString(obj, "cuda_stream");
    if (!h) return false;
    *out = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    return !PyErr_Occurred();
}

// step(q, k, v, alpha, theta, beta, S, o, o_im, stream); step_fused the same with four floats after beta
PyObject *call(PyObject *const *args, Py_ssize_t n, bool fused)
{
    HANDLE_TH_ERRORS
    static const char *const plain[] = {"q", "k", "v", "alpha", "theta", "beta", "S", "o", "o_im"};
    static const char *const raw[] = {"q", "k_raw", "v", "a_raw", "b_raw", "c_raw", "S", "o", "o_im"};
    const char *const *name = fused ? raw : plain;
    const int skip = fused ? 4 : 0;
    if (n != 10 + skip) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    if (!g_step || !g_step_fused) {
        PyErr_SetString(PyExc_RuntimeError, "bind has not been called");
        return nullptr;
    }
    if (!THPVariable_Check(args[0]) || !THPVariable_Check(args[2])) {
        PyErr_SetString(PyExc_TypeError, "q and v must be tensors");
        return nullptr;
    }
    const at::Tensor &q = THPVariable_Unpack(args[0]), &v = THPVariable_Unpack(args[2]);
    if (q.dim() != 3 || v.dim() < 1) {
        PyErr_SetString(PyExc_ValueError, "q must be [B, H, d_k] and v [B, H, d_v]");
        return nullptr;
    }
    const at::ScalarType type = q.scalar_type();
    if (type != at::kFloat && type != at::kBFloat16) {
        PyErr_SetString(PyExc_TypeError, "q, k, v must be float32 or bfloat16");
        return nullptr;
    }
    void *p[9], *stream;
    for (int i = 0; i < 9; ++i) {
        const bool wide = i >= 3 && i <= 6;                       // alpha, theta, beta, S
        if (!address(args[i < 6 ? i : i + skip], name[i], wide ? at::kFloat : type, &p[i])) return nullptr;
    }
    if (!stream_of(args[9 + skip], &stream)) return nullptr;
    const int B = (int)q.size(0), H = (int)q.size(1), dk = (int)q.size(2), dv = (int)v.size(-1), dt = type == at::kBFloat16;
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < skip; ++i) {
        const double x = PyFloat_AsDouble(args[6 + i]);
        if (x == -1.0 && PyErr_Occurred()) return nullptr;
        f[i] = (float)x;
    }
    // The launch runs without the interpreter's lock, as a call through ctypes does: it blocks while the launch queue is
    // full, and what empties the queue may be a host callback that needs the lock.
    int rc;
    Py_BEGIN_ALLOW_THREADS
    const float *alpha = static_cast<const float *>(p[3]), *theta = static_cast<const float *>(p[4]), *beta = static_cast<const float *>(p[5]);
    float *S = static_cast<float *>(p[6]);
    rc = fused ? g_step_fused(p[0], p[1], p[2], alpha, theta, beta, f[0], f[1], f[2], f[3], S, p[7], p[8], B, H, dk, dv, dt, stream)
               : g_step(p[0], p[1], p[2], alpha, theta, beta, S, p[7], p[8], B, H, dk, dv, dt, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

PyObject *step(PyObject *, PyObject *const *args, Py_ssize_t n) { return call(args, n, false); }
PyObject *step_fused(PyObject *, PyObject *const *args, Py_ssize_t n) { return call(args, n, true); }

// bind(address of sfda_step, address of sfda_step_fused)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2) {
        PyErr_SetString(PyExc_TypeError, "bind takes two addresses");
        return nullptr;
    }
    void *a = PyLong_AsVoidPtr(args[0]), *b = PyLong_AsVoidPtr(args[1]);
    if (PyErr_Occurred()) return nullptr;
    g_step = reinterpret_cast<StepFn>(a);
    g_step_fused = reinterpret_cast<StepFusedFn>(b);
    Py_RETURN_NONE;
}

// ---- linear attention with a fixed decay for each head, rotary positions, group norm ------------------------------------
decltype(&sfda_linear_step) g_linear_step = nullptr;
decltype(&sfda_linear_forward) g_linear_forward = nullptr;
decltype(&sfda_linear_backward) g_linear_backward = nullptr;
decltype(&sfda_rotary) g_rotary = nullptr;
decltype(&sfda_group_norm) g_group_norm = nullptr;
decltype(&sfda_group_norm_backward) g_group_norm_backward = nullptr;

// The arguments of one call: positional, all of them given.  A method that fails has set a Python error.
class Args {
  public:
    Args(PyObject *const *args, Py_ssize_t n, Py_ssize_t want) : args_(args), ok_(n == want)
    {
        if (!ok_) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        else if (!g_group_norm_backward) fail(PyExc_RuntimeError, "bind_operators has not been called");
    }
    explicit operator bool() const { return ok_; }
    const at::Tensor *tensor(int i, const char *name)
    {
        if (!ok_) return nullptr;
        if (!THPVariable_Check(args_[i])) return fail(PyExc_TypeError, "%s must be a tensor", name), nullptr;
        return &THPVariable_Unpack(args_[i]);
    }
    // The call's first tensor: it names the element type and the device, which is the current one, whose stream the work goes to.
    const at::Tensor *first(int i, const char *name)
    {
        const at::Tensor *t = tensor(i, name);
        if (!t) return nullptr;
        if (!t->is_cuda()) return fail(PyExc_ValueError, "%s must live on cuda", name), nullptr;
        device_ = t->get_device();
        if (device_ != c10::cuda::current_device()) return fail(PyExc_ValueError, "%s must live on the current device", name), nullptr;
        type_ = t->scalar_type();
        if (type_ != at::kFloat && type_ != at::kBFloat16) return fail(PyExc_TypeError, "%s must be float32 or bfloat16", name), nullptr;
        return t;
    }
    at::ScalarType type() const { return type_; }
    int dtype() const { return type_ == at::kBFloat16 ? SFDA_BF16 : SFDA_F32; }
    bool here(const at::Tensor &t, const char *name, at::ScalarType type)
    {
        if (!t.is_cuda() || t.get_device() != device_) return fail(PyExc_ValueError, "%s must live on the same device as the first tensor", name);
        if (t.scalar_type() != type) {
            const char *is = type == at::kFloat ? "torch.float32" : type == at::kBFloat16 ? "torch.bfloat16" : type == at::kInt ? "torch.int32" : "torch.int64";
            return fail(PyExc_TypeError, "%s must be %s", name, is);
        }
        return true;
    }
    // A dense tensor of this type and shape; NULL for None where that is allowed.
    void *dense(int i, const char *name, at::ScalarType type, at::IntArrayRef shape, bool optional = false)
    {
        if (!ok_ || (optional && args_[i] == Py_None)) return nullptr;
        const at::Tensor *t = tensor(i, name);
        if (!t || !here(*t, name, type)) return nullptr;
        if (!t->is_contiguous()) return fail(PyExc_ValueError, "%s must be contiguous", name), nullptr;
        if (t->sizes() != shape) return fail(PyExc_ValueError, "%s does not have the shape that the other tensors ask for", name), nullptr;
        return t->data_ptr();
    }
    void *scratch(int i, size_t *bytes)
    {
        *bytes = 0;
        if (!ok_ || args_[i] == Py_None) return nullptr;
        const at::Tensor *t = tensor(i, "workspace");
        if (!t) return nullptr;
        if (!t->is_cuda() || t->get_device() != device_ || !t->is_contiguous())
            return fail(PyExc_ValueError, "workspace must be contiguous and live on the same device as the first tensor"), nullptr;
        *bytes = t->nbytes();
        return t->data_ptr();
    }
    float real(int i)
    {
        const double x = ok_ ? PyFloat_AsDouble(args_[i]) : 0.0;
        if (x == -1.0 && PyErr_Occurred()) ok_ = false;
        return (float)x;
    }
    int integer(int i)
    {
        const long x = ok_ ? PyLong_AsLong(args_[i]) : 0;
        if (x == -1 && PyErr_Occurred()) ok_ = false;
        else if (x != (int)x) fail(PyExc_OverflowError, "an integer argument does not fit 32 bits");
        return (int)x;
    }
    bool none(int i) const { return args_[i] == Py_None; }
    void *stream(int i)
    {
        void *s = nullptr;
        if (ok_ && !stream_of(args_[i], &s)) ok_ = false;
        return s;
    }
    bool fail(PyObject *kind, const char *text, const char *name = nullptr, const char *more = nullptr)
    {
        if (ok_) PyErr_Format(kind, text, name, more);
        return ok_ = false;
    }

  private:
    PyObject *const *args_;
    bool ok_;
    int device_ = -1;
    at::ScalarType type_ = at::kFloat;
};

// Runs without the interpreter's lock (see `call`).
template <typename F>
PyObject *launched(F launch)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = launch();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}
const float *f32(void *p) { return static_cast<const float *>(p); }
const int32_t *i32(void *p) { return static_cast<const int32_t *>(p); }

bool fits(Args &a, std::initializer_list<int64_t> sizes)
{
    for (const int64_t n : sizes)
        if (n > 0x7fffffff) return a.fail(PyExc_ValueError, "a dimension does not fit 32 bits");
    return true;
}

// linear_step(q, k, v, log_decay, S, o, scale, stream)
PyObject *linear_step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a(args, n, 8);
    const at::Tensor *q = a.first(0, "q"), *v = a.tensor(2, "v");
    if (!a) return nullptr;
    if (q->dim() != 3 || v->dim() != 3) return a.fail(PyExc_ValueError, "q must be [B, H, d_k], k [B, H_kv, d_k] and v [B, H_kv, d_v]"), nullptr;
    const int64_t B = q->size(0), H = q->size(1), dk = q->size(2), Hk = v->size(1), dv = v->size(2);
    void *pq = a.dense(0, "q", a.type(), {B, H, dk}), *pk = a.dense(1, "k", a.type(), {B, Hk, dk}), *pv = a.dense(2, "v", a.type(), {B, Hk, dv});
    void *ld = a.dense(3, "log_decay", at::kFloat, {H}), *S = a.dense(4, "S", at::kFloat, {B, H, dk, dv}), *o = a.dense(5, "o", a.type(), {B, H, dv});
    const float scale = a.real(6);
    void *stream = a.stream(7);
    if (!a || !fits(a, {B, H})) return nullptr;
    return launched([&] { return g_linear_step(pq, pk, pv, f32(ld), static_cast<float *>(S), o, (int)B, (int)H, (int)Hk, (int)dk, (int)dv, a.dtype(), scale, stream); });
    END_HANDLE_TH_ERRORS
}

// The tensors that the forward and its gradients share, at places 0..7: q, k, v, log_decay, lens, S0, o (d_o), S_T (dS_T)
struct Sequences {
    int64_t B = 0, T = 0, H = 0, Hk = 0, dk = 0, dv = 0;
    void *p[8] = {};
    Sequences(Args &a, bool backward)
    {
        const at::Tensor *q = a.first(0, "q"), *v = a.tensor(2, "v");
        if (!a) return;
        if (q->dim() != 4 || v->dim() != 4) {
            a.fail(PyExc_ValueError, "q must be [B, T, H, d_k], k [B, T, H_kv, d_k] and v [B, T, H_kv, d_v]");
            return;
        }
        B = q->size(0); T = q->size(1); H = q->size(2); dk = q->size(3); Hk = v->size(2); dv = v->size(3);
        p[0] = a.dense(0, "q", a.type(), {B, T, H, dk});
        p[1] = a.dense(1, "k", a.type(), {B, T, Hk, dk});
        p[2] = a.dense(2, "v", a.type(), {B, T, Hk, dv});
        p[3] = a.dense(3, "log_decay", at::kFloat, {H});
        p[4] = a.dense(4, "lens", at::kInt, {B}, true);
        p[5] = a.dense(5, "S0", at::kFloat, {B, H, dk, dv}, true);
        p[6] = a.dense(6, backward ? "d_o" : "o", a.type(), {B, T, H, dv});
        p[7] = a.dense(7, backward ? "dS_T" : "S_T", at::kFloat, {B, H, dk, dv}, true);
        if (a) fits(a, {B, T, H});
    }
};

// linear_forward(q, k, v, log_decay, lens, S0, o, S_T, scale, workspace, stream)
PyObject *linear_forward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a(args, n, 11);
    const Sequences s(a, false);
    const float scale = a ? a.real(8) : 0.f;
    size_t bytes;
    void *ws = a.scratch(9, &bytes), *stream = a.stream(10);
    if (!a) return nullptr;
    return launched([&] {
        return g_linear_forward(s.p[0], s.p[1], s.p[2], f32(s.p[3]), i32(s.p[4]), f32(s.p[5]), s.p[6], static_cast<float *>(s.p[7]), (int)s.B, (int)s.T,
                                (int)s.H, (int)s.Hk, (int)s.dk, (int)s.dv, a.dtype(), scale, ws, bytes, stream);
    });
    END_HANDLE_TH_ERRORS
}

// linear_backward(q, k, v, log_decay, lens, S0, d_o, dS_T, dq, dk, dv, dS0, scale, workspace, stream)
PyObject *linear_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a(args, n, 15);
    const Sequences s(a, true);
    void *dq = a.dense(8, "dq", a.type(), {s.B, s.T, s.H, s.dk}), *dk = a.dense(9, "dk", a.type(), {s.B, s.T, s.Hk, s.dk});
    void *dv = a.dense(10, "dv", a.type(), {s.B, s.T, s.Hk, s.dv}), *dS0 = a.dense(11, "dS0", at::kFloat, {s.B, s.H, s.dk, s.dv});
    const float scale = a ? a.real(12) : 0.f;
    size_t bytes;
    void *ws = a.scratch(13, &bytes), *stream = a.stream(14);
    if (!a) return nullptr;
    return launched([&] {
        return g_linear_backward(s.p[0], s.p[1], s.p[2], f32(s.p[3]), i32(s.p[4]), f32(s.p[5]), s.p[6], f32(s.p[7]), dq, dk, dv, static_cast<float *>(dS0),
                                 (int)s.B, (int)s.T, (int)s.H, (int)s.Hk, (int)s.dk, (int)s.dv, a.dtype(), scale, ws, bytes, stream);
    });
    END_HANDLE_TH_ERRORS
}

// [B, T, heads, d] or [B, heads, d] with dense heads and one stride from token to token: that stride in elements
bool rows_of(Args &a, int i, const char *name, const at::Tensor &like, const at::Tensor **out, int64_t *stride)
{
    const at::Tensor *t = a.tensor(i, name);
    if (!t || !a.here(*t, name, a.type())) return false;
    const int64_t dim = t->dim(), like_dim = like.dim();
    if (dim != 3 && dim != 4) return a.fail(PyExc_ValueError, "%s must be [B, T, heads, d] or [B, heads, d]", name);
    bool same = dim == like_dim && t->size(dim - 1) == like.size(dim - 1);
    for (int64_t x = 0; same && x < dim - 2; ++x) same = t->size(x) == like.size(x);
    if (!same) return a.fail(PyExc_ValueError, "%s does not have the tokens and channels of the other tensors", name);
    const int64_t d = t->size(dim - 1), h = t->size(dim - 2);
    if ((d > 1 && t->stride(dim - 1) != 1) || (h > 1 && t->stride(dim - 2) != d)) return a.fail(PyExc_ValueError, "%s must have dense heads", name);
    *stride = h * d;
    if (dim == 3) {
        if (t->size(0) > 1) *stride = t->stride(0);
    } else if (t->size(1) > 1) {
        *stride = t->stride(1);
        if (t->size(0) > 1 && t->stride(0) != t->size(1) * *stride) return a.fail(PyExc_ValueError, "%s must have one stride from token to token", name);
    } else if (t->size(0) > 1) {
        *stride = t->stride(0);
    }
    *out = t;
    return true;
}

// rotary(q, k, positions, turns, q_out, k_out, layout, amplitude, inverse, stream)
PyObject *rotary(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a(args, n, 10);
    const at::Tensor *q = a.first(0, "q"), *k = nullptr, *qo = nullptr, *ko = nullptr;
    if (!a) return nullptr;
    int64_t sq = 0, sk = 0, sqo = 0, sko = 0;
    if (!rows_of(a, 0, "q", *q, &q, &sq) || !rows_of(a, 4, "q_out", *q, &qo, &sqo)) return nullptr;
    if (qo->sizes() != q->sizes()) return a.fail(PyExc_ValueError, "q_out must have the shape of q"), nullptr;
    if (a.none(1) != a.none(5)) return a.fail(PyExc_TypeError, "k and k_out go together"), nullptr;
    if (!a.none(1)) {
        if (!rows_of(a, 1, "k", *q, &k, &sk) || !rows_of(a, 5, "k_out", *q, &ko, &sko)) return nullptr;
        if (ko->sizes() != k->sizes()) return a.fail(PyExc_ValueError, "k_out must have the shape of k"), nullptr;
    }
    const int64_t dim = q->dim(), B = q->size(0), T = dim == 4 ? q->size(1) : 1;
    const at::Tensor *pos = a.tensor(2, "positions"), *turns = a.tensor(3, "turns");
    if (!a) return nullptr;
    void *pp = dim == 4 || pos->dim() == 2 ? a.dense(2, "positions", at::kInt, {B, T}) : a.dense(2, "positions", at::kInt, {B});
    void *pt = a.dense(3, "turns", at::kLong, {turns->numel()});
    const int layout = a.integer(6);
    const float amplitude = a.real(7);
    const int inverse = a ? PyObject_IsTrue(args[8]) : 0;
    void *stream = a.stream(9);
    if (!a || inverse < 0 || !fits(a, {B, T, q->size(dim - 2), q->size(dim - 1), 2 * turns->numel()})) return nullptr;
    return launched([&] {
        return g_rotary(q->data_ptr(), k ? k->data_ptr() : nullptr, i32(pp), static_cast<const uint64_t *>(pt), qo->data_ptr(), ko ? ko->data_ptr() : nullptr,
                        (int)B, (int)T, (int)q->size(dim - 2), k ? (int)k->size(dim - 2) : 0, (int)q->size(dim - 1), (int)(2 * turns->numel()), sq, sk, sqo,
                        sko, layout, amplitude, inverse, a.dtype(), stream);
    });
    END_HANDLE_TH_ERRORS
}

// group_norm(x, weight, bias, gate, y, groups, eps, act, stream)
PyObject *group_norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a(args, n, 9);
    const at::Tensor *x = a.first(0, "x");
    if (!a) return nullptr;
    if (x->dim() < 1 || x->numel() == 0) return a.fail(PyExc_ValueError, "x must be [..., C] with at least one row"), nullptr;
    const int64_t C = x->size(-1), rows = x->numel() / C;
    void *px = a.dense(0, "x", a.type(), x->sizes()), *w = a.dense(1, "weight", at::kFloat, {C}, true), *b = a.dense(2, "bias", at::kFloat, {C}, true);
    void *gate = a.dense(3, "gate", a.type(), x->sizes(), true), *y = a.dense(4, "y", a.type(), x->sizes());
    const int groups = a.integer(5), act = a.integer(7);
    const float eps = a.real(6);
    void *stream = a.stream(8);
    if (!a || !fits(a, {C})) return nullptr;
    return launched([&] { return g_group_norm(px, f32(w), f32(b), gate, y, rows, (int)C, groups, eps, act, a.dtype(), stream); });
    END_HANDLE_TH_ERRORS
}

// group_norm_backward(x, weight, bias, gate, dy, dx, dweight, dbias, dgate, groups, eps, act, workspace, stream)
PyObject *group_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    Args a(args, n, 14);
    const at::Tensor *x = a.first(0, "x");
    if (!a) return nullptr;
    if (x->dim() < 1 || x->numel() == 0) return a.fail(PyExc_ValueError, "x must be [..., C] with at least one row"), nullptr;
    const int64_t C = x->size(-1), rows = x->numel() / C;
    void *px = a.dense(0, "x", a.type(), x->sizes()), *w = a.dense(1, "weight", at::kFloat, {C}, true), *b = a.dense(2, "bias", at::kFloat, {C}, true);
    void *gate = a.dense(3, "gate", a.type(), x->sizes(), true), *dy = a.dense(4, "dy", a.type(), x->sizes()), *dx = a.dense(5, "dx", a.type(), x->sizes());
    void *dw = a.dense(6, "dweight", at::kFloat, {C}, true), *db = a.dense(7, "dbias", at::kFloat, {C}, true);
    void *dgate = a.dense(8, "dgate", a.type(), x->sizes(), gate == nullptr);
    const int groups = a.integer(9), act = a.integer(11);
    const float eps = a.real(10);
    size_t bytes;
    void *ws = a.scratch(12, &bytes), *stream = a.stream(13);
    if (!a || !fits(a, {C})) return nullptr;
    return launched([&] {
        return g_group_norm_backward(px, f32(w), f32(b), gate, dy, dx, static_cast<float *>(dw), static_cast<float *>(db), dgate, rows, (int)C, groups, eps, act,
                                     a.dtype(), ws, bytes, stream);
    });
    END_HANDLE_TH_ERRORS
}

// bind_operators(addresses of sfda_linear_step, _forward, _backward, sfda_rotary, sfda_group_norm, _backward)
PyObject *bind_operators(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "bind_operators takes six addresses");
        return nullptr;
    }
    void *p[6];
    for (int i = 0; i < 6; ++i) p[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    g_linear_step = reinterpret_cast<decltype(g_linear_step)>(p[0]);
    g_linear_forward = reinterpret_cast<decltype(g_linear_forward)>(p[1]);
    g_linear_backward = reinterpret_cast<decltype(g_linear_backward)>(p[2]);
    g_rotary = reinterpret_cast<decltype(g_rotary)>(p[3]);
    g_group_norm = reinterpret_cast<decltype(g_group_norm)>(p[4]);
    g_group_norm_backward = reinterpret_cast<decltype(g_group_norm_backward)>(p[5]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         {"step", (PyCFunction)(void (*)(void))step, METH_FASTCALL, nullptr},
                         {"step_fused", (PyCFunction)(void (*)(void))step_fused, METH_FASTCALL, nullptr},
                         {"bind_operators", (PyCFunction)(void (*)(void))bind_operators, METH_FASTCALL, nullptr},
                         {"linear_step", (PyCFunction)(void (*)(void))linear_step, METH_FASTCALL, nullptr},
                         {"linear_forward", (PyCFunction)(void (*)(void))linear_forward, METH_FASTCALL, nullptr},
                         {"linear_backward", (PyCFunction)(void (*)(void))linear_backward, METH_FASTCALL, nullptr},
                         {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
                         {"group_norm", (PyCFunction)(void (*)(void))group_norm, METH_FASTCALL, nullptr},
                         {"group_norm_backward", (PyCFunction)(void (*)(void))group_norm_backward, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__host(void) { return PyModule_Create(&module); }
