// Host path of the per-call entry points: a CPython module that takes the binding's arguments as they are (the configuration, tensors,
// numbers), checks them and calls the C ABI on the current stream.  Through ctypes the same work is 12 to 20 interpreted attribute reads and the
// conversion of every argument: 2.7 us of a call beside the 2.6 us of its launch, more than the kernels of a small call take.
//
// A function returns the library's status when it has made the call, and -1, with nothing done, for every argument that is not of the
// ordinary kind (no buffer given, another type, tensor subclasses and wrapped tensors, an active torch-function mode, of which
// torch.set_default_device is one, a failed check); the binding then goes through its own checks and ctypes, which raise what they raise.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "lq.h"

namespace {

constexpr int NOT_HERE = -1;
PyTypeObject* config_type = nullptr;  // binding.lq_config, a ctypes.Structure laid out as lq_config
PyTypeObject *adapter_config_type = nullptr, *qk_config_type = nullptr;  // binding.lq_adapter_config, binding.lq_qk_config

// An ordinary GPU tensor: exactly torch.Tensor or Parameter, strided, with memory of its own.
const at::Tensor* tensor(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != c10::kStrided || !t.has_storage()) return nullptr;
    if (t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                                 c10::DispatchKey::Functionalize, c10::DispatchKey::Python})))
        return nullptr;
    return &t;
}
bool dense(const at::Tensor* t, c10::ScalarType ty, int64_t rows, int64_t cols)  // contiguous rows x cols
{
    return t && t->scalar_type() == ty && t->dim() == 2 && t->size(0) == rows && t->size(1) == cols && t->is_contiguous();
}
bool row_major(const at::Tensor* t, c10::ScalarType ty, int64_t cols)  // rows may be further apart than cols
{
    return t && t->scalar_type() == ty && t->dim() == 2 && t->stride(1) == 1 && t->size(1) == cols;
}
bool integer(PyObject* o, int64_t* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
bool number(PyObject* o, float* v)
{
    if (!PyFloat_CheckExact(o)) return false;
    *v = (float)PyFloat_AS_DOUBLE(o);
    return true;
}

// A configuration's bytes, held for the duration of a call.
template <typename T>
struct ConfigOf {
    Py_buffer view{};
    const T* p = nullptr;
    ConfigOf(PyObject* o, PyTypeObject* type)
    {
        if (!type || Py_TYPE(o) != type) return;
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            return;
        }
        if (view.len == (Py_ssize_t)sizeof(T)) p = (const T*)view.buf;
    }
    ~ConfigOf()
    {
        if (view.obj) PyBuffer_Release(&view);
    }
    ConfigOf(const ConfigOf&) = delete;
    ConfigOf& operator=(const ConfigOf&) = delete;
};
struct Config : ConfigOf<lq_config> {
    explicit Config(PyObject* o) : ConfigOf(o, config_type) {}
};

// Runs f (which returns a status, or NOT_HERE before it has called anything) for n arguments; a C++ exception is NOT_HERE as well: only
// the tensors' accessors throw, all of them before the call.
template <typename F>
PyObject* guarded(Py_ssize_t nargs, Py_ssize_t n, F f)
{
    int st = NOT_HERE;
    if (nargs == n && !at::impl::torch_function_mode_enabled()) {
        try {
            st = f();
        } catch (...) {
            st = NOT_HERE;
        }
    }
    return PyLong_FromLong(st);
}
template <typename F>
int on_stream(F call)  // the launch without the interpreter lock, as ctypes makes it
{
    void* s = (void*)c10::hip::getCurrentHIPStream().stream();
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = (int)call(s);
    Py_END_ALLOW_THREADS
    return st;
}

PyObject* set_config_type(PyObject*, PyObject* type)
{
    if (!PyType_Check(type)) {
        PyErr_SetString(PyExc_TypeError, "a type is needed");
        return nullptr;
    }
    Py_INCREF(type);
    Py_XDECREF((PyObject*)config_type);
    config_type = (PyTypeObject*)type;
    Py_RETURN_NONE;
}

PyObject* quantize_act(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, packed, X, act
{
    return guarded(n, 4, [&] {
        const Config c(a[0]);
        const at::Tensor *packed = tensor(a[1]), *X = tensor(a[2]), *act = tensor(a[3]);
        if (!c.p || !packed || !act || !row_major(X, c.p->x_dtype == LQ_BF16 ? at::kBFloat16 : at::kFloat, c.p->K) || X->size(0) == 0) return NOT_HERE;
        const void *pp = packed->data_ptr(), *xp = X->data_ptr();
        void* ap = act->data_ptr();
        const int64_t pn = packed->numel(), M = X->size(0), ld = X->stride(0), an = act->numel();
        return on_stream([&](void* s) { return lq_quantize_act(c.p, pp, (size_t)pn, xp, M, ld, ap, (size_t)an, nullptr, s); });
    });
}

PyObject* linear_lowrank_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, packed, act, M, Y
{
    return guarded(n, 5, [&] {
        const Config c(a[0]);
        const at::Tensor *packed = tensor(a[1]), *act = tensor(a[2]), *Y = tensor(a[4]);
        int64_t M;
        if (!c.p || !packed || !act || !integer(a[3], &M) || !row_major(Y, at::kBFloat16, c.p->N) || Y->size(0) != M) return NOT_HERE;
        const void *pp = packed->data_ptr(), *ap = act->data_ptr();
        void* yp = Y->data_ptr();
        const int64_t pn = packed->numel(), an = act->numel(), ld = Y->stride(0);
        return on_stream([&](void* s) { return lq_linear_lowrank_fwd(c.p, pp, (size_t)pn, ap, (size_t)an, M, yp, ld, nullptr, s); });
    });
}

PyObject* linear_lowrank_fwd_handoff(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, packed, act, M, next_cfg, act_next, codes, Y or None
{
    return guarded(n, 8, [&] {
        const Config c(a[0]), cn(a[4]);
        const at::Tensor *packed = tensor(a[1]), *act = tensor(a[2]), *next = tensor(a[5]), *codes = tensor(a[6]);
        const at::Tensor* Y = a[7] == Py_None ? nullptr : tensor(a[7]);
        int64_t M;
        if (!c.p || !cn.p || !packed || !act || !next || !codes || !integer(a[3], &M)) return NOT_HERE;
        if (a[7] != Py_None && (!row_major(Y, at::kBFloat16, c.p->N) || Y->size(0) != M)) return NOT_HERE;
        const void *pp = packed->data_ptr(), *ap = act->data_ptr();
        void *np = next->data_ptr(), *cp = codes->data_ptr(), *yp = Y ? Y->data_ptr() : nullptr;
        const int64_t pn = packed->numel(), an = act->numel(), nn = next->numel(), kn = codes->numel(), ld = Y ? Y->stride(0) : 0;
        return on_stream([&](void* s) {
            return lq_linear_lowrank_fwd_handoff(c.p, pp, (size_t)pn, ap, (size_t)an, M, yp, ld, cn.p, np, (size_t)nn, cp, (size_t)kn, s);
        });
    });
}

PyObject* branch_from_codes(PyObject*, PyObject* const* a, Py_ssize_t n)  // next_cfg, packed_next, codes, M, act_next
{
    return guarded(n, 5, [&] {
        const Config c(a[0]);
        const at::Tensor *packed = tensor(a[1]), *codes = tensor(a[2]), *act = tensor(a[4]);
        int64_t M;
        if (!c.p || !packed || !codes || !act || !integer(a[3], &M)) return NOT_HERE;
        const void *pp = packed->data_ptr(), *cp = codes->data_ptr();
        void* ap = act->data_ptr();
        const int64_t pn = packed->numel(), kn = codes->numel(), an = act->numel();
        return on_stream([&](void* s) { return lq_branch_from_codes(c.p, pp, (size_t)pn, cp, (size_t)kn, M, ap, (size_t)an, s); });
    });
}

PyObject* pack_weights(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, W, L, R, packed
{
    return guarded(n, 5, [&] {
        const Config c(a[0]);
        const at::Tensor *W = tensor(a[1]), *L = tensor(a[2]), *R = tensor(a[3]), *packed = tensor(a[4]);
        if (!c.p || !packed || !dense(W, at::kFloat, c.p->N, c.p->K) || !dense(L, at::kFloat, c.p->N, c.p->rank) || !dense(R, at::kFloat, c.p->rank, c.p->K))
            return NOT_HERE;
        const float *wp = (const float*)W->data_ptr(), *lp = (const float*)L->data_ptr(), *rp = (const float*)R->data_ptr();
        void* pp = packed->data_ptr();
        const int64_t pn = packed->numel();
        return on_stream([&](void* s) { return lq_pack_weights(c.p, wp, lp, rp, pp, (size_t)pn, s); });
    });
}

bool loss_arg(PyObject* o, void** p)
{
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = tensor(o);
    if (!t) return false;
    *p = t->data_ptr();
    return true;
}

PyObject* calib_step(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, W, state, step, lr, beta1, beta2, eps, loss or None
{
    return guarded(n, 9, [&] {
        const Config c(a[0]);
        const at::Tensor *W = tensor(a[1]), *state = tensor(a[2]);
        int64_t step;
        lq_adam ad;
        void* loss;
        if (!c.p || !state || !dense(W, at::kFloat, c.p->N, c.p->K) || !integer(a[3], &step) || step < INT32_MIN || step > INT32_MAX) return NOT_HERE;
        if (!number(a[4], &ad.lr) || !number(a[5], &ad.beta1) || !number(a[6], &ad.beta2) || !number(a[7], &ad.eps) || !loss_arg(a[8], &loss)) return NOT_HERE;
        const float* wp = (const float*)W->data_ptr();
        void* sp = state->data_ptr();
        const int64_t sn = state->numel();
        return on_stream([&](void* s) { return lq_calib_step(c.p, wp, sp, (size_t)sn, (int32_t)step, &ad, (float*)loss, s); });
    });
}

PyObject* rot_step(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, L, R, state, lr, beta, eps, q, s, grad_scale, loss or None
{
    return guarded(n, 11, [&] {
        const Config c(a[0]);
        const at::Tensor *L = tensor(a[1]), *R = tensor(a[2]), *state = tensor(a[3]);
        int64_t passes;
        lq_cayley cs;
        void* loss;
        if (!c.p || !state || !dense(L, at::kFloat, c.p->N, c.p->rank) || !dense(R, at::kFloat, c.p->rank, c.p->K)) return NOT_HERE;
        if (!number(a[4], &cs.lr) || !number(a[5], &cs.beta) || !number(a[6], &cs.eps) || !number(a[7], &cs.q) || !integer(a[8], &passes) ||
            passes < INT32_MIN || passes > INT32_MAX || !number(a[9], &cs.grad_scale) || !loss_arg(a[10], &loss))
            return NOT_HERE;
        cs.s = (int32_t)passes;
        const float *lp = (const float*)L->data_ptr(), *rp = (const float*)R->data_ptr();
        void* sp = state->data_ptr();
        const int64_t sn = state->numel();
        return on_stream([&](void* s) { return lq_rot_step(c.p, lp, rp, sp, (size_t)sn, &cs, (float*)loss, s); });
    });
}

PyObject* set_operator_config_types(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != 2 || !PyType_Check(a[0]) || !PyType_Check(a[1])) {
        PyErr_SetString(PyExc_TypeError, "two types are needed");
        return nullptr;
    }
    Py_INCREF(a[0]);
    Py_INCREF(a[1]);
    Py_XDECREF((PyObject*)adapter_config_type);
    Py_XDECREF((PyObject*)qk_config_type);
    adapter_config_type = (PyTypeObject*)a[0];
    qk_config_type = (PyTypeObject*)a[1];
    Py_RETURN_NONE;
}

bool blob(const at::Tensor* t) { return t && t->scalar_type() == at::kByte && t->is_contiguous(); }
bool vec(const at::Tensor* t, c10::ScalarType ty, int64_t n) { return t && t->scalar_type() == ty && t->numel() == n && t->is_contiguous(); }
bool cube(const at::Tensor* t, c10::ScalarType ty, int64_t a, int64_t b, int64_t c)
{
    return t && t->scalar_type() == ty && t->dim() == 3 && t->size(0) == a && t->size(1) == b && t->size(2) == c && t->is_contiguous();
}
bool rows(const at::Tensor* t, c10::ScalarType ty, int64_t M, int64_t cols) { return row_major(t, ty, cols) && t->size(0) == M; }
int64_t row_stride(const at::Tensor* t)  // of a single row: its length
{
    return t->size(0) > 1 || t->stride(0) > t->size(1) ? t->stride(0) : t->size(1);
}
bool optional(PyObject* o, const at::Tensor** t)  // None, or an ordinary tensor
{
    *t = nullptr;
    if (o == Py_None) return true;
    *t = tensor(o);
    return *t != nullptr;
}

PyObject* adapter_plan(PyObject*, PyObject* const* a, Py_ssize_t n)  // slots, ids, plan
{
    return guarded(n, 3, [&] {
        int64_t slots;
        const at::Tensor *ids = tensor(a[1]), *plan = tensor(a[2]);
        if (!integer(a[0], &slots) || slots < INT32_MIN || slots > INT32_MAX || !ids || ids->scalar_type() != at::kInt || ids->dim() != 1 ||
            !ids->is_contiguous() || !blob(plan))
            return NOT_HERE;
        const int32_t* ip = (const int32_t*)ids->data_ptr();
        void* pp = plan->data_ptr();
        const int64_t M = ids->size(0), pn = plan->numel();
        return on_stream([&](void* s) { return lq_adapter_plan((int32_t)slots, ip, M, pp, (size_t)pn, s); });
    });
}

// A, B, ranks, scales at a[0..3]
bool pool_arg(const lq_adapter_config* c, PyObject* const* a, lq_adapter_pool* p)
{
    const at::Tensor *A = tensor(a[0]), *B = tensor(a[1]), *ranks = tensor(a[2]), *scales = tensor(a[3]);
    if (!cube(A, at::kBFloat16, c->slots, c->rank, c->K) || !cube(B, at::kBFloat16, c->slots, c->N, c->rank) || !vec(ranks, at::kInt, c->slots) ||
        !vec(scales, at::kFloat, c->slots) || ranks->dim() != 1 || scales->dim() != 1)
        return false;
    *p = {A->data_ptr(), B->data_ptr(), (const int32_t*)ranks->data_ptr(), (const float*)scales->data_ptr()};
    return true;
}

PyObject* adapter_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, plan, X, A, B, ranks, scales, Yin, Y, inter
{
    return guarded(n, 10, [&] {
        const ConfigOf<lq_adapter_config> c(a[0], adapter_config_type);
        const at::Tensor *plan = tensor(a[1]), *X = tensor(a[2]), *Yin = tensor(a[7]), *Y = tensor(a[8]), *inter = tensor(a[9]);
        lq_adapter_pool pool;
        if (!c.p || !blob(plan) || !blob(inter) || !row_major(X, c.p->x_dtype == LQ_BF16 ? at::kBFloat16 : at::kFloat, c.p->K) || !pool_arg(c.p, a + 3, &pool))
            return NOT_HERE;
        const int64_t M = X->size(0);
        if (!rows(Yin, at::kBFloat16, M, c.p->N) || !rows(Y, at::kBFloat16, M, c.p->N)) return NOT_HERE;
        const void *pp = plan->data_ptr(), *xp = X->data_ptr(), *yi = Yin->data_ptr();
        void *yp = Y->data_ptr(), *ip = inter->data_ptr();
        const int64_t pn = plan->numel(), in = inter->numel(), lx = row_stride(X), li = row_stride(Yin), ly = row_stride(Y);
        return on_stream([&](void* s) { return lq_adapter_fwd(c.p, pp, (size_t)pn, &pool, xp, lx, yi, li, yp, ly, M, ip, (size_t)in, s); });
    });
}

PyObject* adapter_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, plan, X, A, B, ranks, scales, inter, dY, dXin or None, dX, dA, dB, work
{
    return guarded(n, 14, [&] {
        const ConfigOf<lq_adapter_config> c(a[0], adapter_config_type);
        const at::Tensor *plan = tensor(a[1]), *X = tensor(a[2]), *inter = tensor(a[7]), *dY = tensor(a[8]), *dXin, *dX = tensor(a[10]), *dA = tensor(a[11]),
                         *dB = tensor(a[12]), *work = tensor(a[13]);
        lq_adapter_pool pool;
        if (!c.p || !blob(plan) || !blob(inter) || !blob(work) || !optional(a[9], &dXin)) return NOT_HERE;
        const c10::ScalarType xt = c.p->x_dtype == LQ_BF16 ? at::kBFloat16 : at::kFloat;
        if (!row_major(X, xt, c.p->K) || !pool_arg(c.p, a + 3, &pool)) return NOT_HERE;
        const int64_t M = X->size(0);
        if (!rows(dY, at::kBFloat16, M, c.p->N) || !rows(dX, xt, M, c.p->K) || (dXin && !rows(dXin, xt, M, c.p->K)) ||
            !cube(dA, at::kFloat, c.p->slots, c.p->rank, c.p->K) || !cube(dB, at::kFloat, c.p->slots, c.p->N, c.p->rank))
            return NOT_HERE;
        const void *pp = plan->data_ptr(), *xp = X->data_ptr(), *ip = inter->data_ptr(), *gy = dY->data_ptr(), *gi = dXin ? dXin->data_ptr() : nullptr;
        void *gx = dX->data_ptr(), *wp = work->data_ptr();
        float *ap = (float*)dA->data_ptr(), *bp = (float*)dB->data_ptr();
        const int64_t pn = plan->numel(), in = inter->numel(), wn = work->numel(), lx = row_stride(X), ly = row_stride(dY), li = dXin ? row_stride(dXin) : 0,
                      lg = row_stride(dX);
        return on_stream([&](void* s) {
            return lq_adapter_bwd(c.p, pp, (size_t)pn, &pool, xp, lx, ip, (size_t)in, gy, ly, gi, li, gx, lg, ap, bp, M, wp, (size_t)wn, s);
        });
    });
}

// Heads of M tokens, or nothing where there are none of the kind.
bool heads_arg(const lq_qk_config* c, PyObject* o, int64_t M, int heads, lq_heads* h)
{
    *h = {nullptr, 0, 0};
    if (heads == 0) return true;
    const at::Tensor* t = tensor(o);
    if (!t || t->scalar_type() != (c->dtype == LQ_BF16 ? at::kBFloat16 : at::kFloat) || t->dim() != 3 || t->size(0) != M || t->size(1) != heads ||
        t->size(2) != c->head_dim || t->stride(2) != 1)
        return false;
    *h = {t->data_ptr(), t->stride(0), t->stride(1)};
    return true;
}
struct QkVectors {
    const float *wq = nullptr, *wk = nullptr, *pos = nullptr, *inv_freq = nullptr;
    int64_t pos_rows = 0;
};
// wq, wk, pos, inv_freq at a[0..3]
bool qk_vectors(const lq_qk_config* c, PyObject* const* a, QkVectors* v)
{
    const at::Tensor *wq, *wk;
    if (!optional(a[0], &wq) || !optional(a[1], &wk) || (wq && !vec(wq, at::kFloat, c->head_dim)) || (wk && !vec(wk, at::kFloat, c->head_dim))) return false;
    v->wq = wq ? (const float*)wq->data_ptr() : nullptr;
    v->wk = wk ? (const float*)wk->data_ptr() : nullptr;
    const int64_t P = (int64_t)c->pairs[0] + c->pairs[1] + c->pairs[2] + c->pairs[3];
    if (P == 0) return true;
    const at::Tensor *pos = tensor(a[2]), *f = tensor(a[3]);
    if (!pos || pos->scalar_type() != at::kFloat || pos->dim() != 2 || pos->size(1) != c->axes || !pos->is_contiguous() || !vec(f, at::kFloat, P)) return false;
    v->pos = (const float*)pos->data_ptr();
    v->inv_freq = (const float*)f->data_ptr();
    v->pos_rows = pos->size(0);
    return true;
}
bool qk_tokens(const lq_qk_config* c, PyObject* q, PyObject* k, int64_t* M)
{
    const at::Tensor* t = tensor(c->heads_q ? q : k);
    if (!t || t->dim() != 3) return false;
    *M = t->size(0);
    return true;
}

PyObject* qk_norm_rope_fwd(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, q, k, wq, wk, pos, inv_freq, qo, ko
{
    return guarded(n, 9, [&] {
        const ConfigOf<lq_qk_config> c(a[0], qk_config_type);
        int64_t M;
        QkVectors v;
        lq_heads h[4];
        if (!c.p || !qk_tokens(c.p, a[1], a[2], &M) || !qk_vectors(c.p, a + 3, &v) || !heads_arg(c.p, a[1], M, c.p->heads_q, &h[0]) ||
            !heads_arg(c.p, a[2], M, c.p->heads_k, &h[1]) || !heads_arg(c.p, a[7], M, c.p->heads_q, &h[2]) || !heads_arg(c.p, a[8], M, c.p->heads_k, &h[3]))
            return NOT_HERE;
        return on_stream([&](void* s) { return lq_qk_norm_rope_fwd(c.p, &h[0], &h[1], v.wq, v.wk, v.pos, v.pos_rows, v.inv_freq, &h[2], &h[3], M, s); });
    });
}

PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* a, Py_ssize_t n)  // cfg, q, k, wq, wk, pos, inv_freq, dqo, dko, dq, dk, dwq, dwk, work
{
    return guarded(n, 14, [&] {
        const ConfigOf<lq_qk_config> c(a[0], qk_config_type);
        int64_t M;
        QkVectors v;
        lq_heads h[6] = {};
        const at::Tensor *dwq, *dwk, *work;
        if (!c.p || !qk_tokens(c.p, a[7], a[8], &M) || !qk_vectors(c.p, a + 3, &v) || !heads_arg(c.p, a[7], M, c.p->heads_q, &h[2]) ||
            !heads_arg(c.p, a[8], M, c.p->heads_k, &h[3]) || !heads_arg(c.p, a[9], M, c.p->heads_q, &h[4]) || !heads_arg(c.p, a[10], M, c.p->heads_k, &h[5]) ||
            !optional(a[11], &dwq) || !optional(a[12], &dwk) || !optional(a[13], &work))
            return NOT_HERE;
        const bool norm = c.p->norm == LQ_NORM_RMS;
        if (norm && (!heads_arg(c.p, a[1], M, c.p->heads_q, &h[0]) || !heads_arg(c.p, a[2], M, c.p->heads_k, &h[1]) || !vec(dwq, at::kFloat, c.p->head_dim) ||
                     !vec(dwk, at::kFloat, c.p->head_dim) || !blob(work)))
            return NOT_HERE;
        float *pq = norm ? (float*)dwq->data_ptr() : nullptr, *pk = norm ? (float*)dwk->data_ptr() : nullptr;
        void* wp = norm ? work->data_ptr() : nullptr;
        const int64_t wn = norm ? work->numel() : 0;
        return on_stream([&](void* s) {
            return lq_qk_norm_rope_bwd(c.p, &h[0], &h[1], v.wq, v.wk, v.pos, v.pos_rows, v.inv_freq, &h[2], &h[3], &h[4], &h[5], pq, pk, M, wp, (size_t)wn, s);
        });
    });
}

#define FAST(NAME) {#NAME, (PyCFunction)(void (*)(void))NAME, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"set_config_type", set_config_type, METH_O, nullptr},
                         FAST(quantize_act),
                         FAST(linear_lowrank_fwd),
                         FAST(linear_lowrank_fwd_handoff),
                         FAST(branch_from_codes),
                         FAST(pack_weights),
                         FAST(calib_step),
                         FAST(rot_step),
                         FAST(set_operator_config_types),
                         FAST(adapter_plan),
                         FAST(adapter_fwd),
                         FAST(adapter_bwd),
                         FAST(qk_norm_rope_fwd),
                         FAST(qk_norm_rope_bwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module); }
