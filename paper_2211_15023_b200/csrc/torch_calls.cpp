// Python entry of the hot calls: what binding.py would do for every Actor step -- check the tensors,
// allocate the results, find the current stream, call the C ABI -- in native code.  At the small
// batches of a single Actor the step is bound by exactly this host work: the CartPole step at batch
// 160 took 15.0 us through ctypes and torch's Python functions, of which the GPU needed five.
//
// Every function returns the results, the status code (an int) of a call that failed, or None when
// the arguments are not what the fast path takes (binding.py then checks them one by one, raises for what a
// kernel could not read, and goes through ctypes with the rest).
#include <Python.h>

#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <optional>

#include "accerl.h"

namespace {

// a CUDA tensor of the given type whose elements are contiguous, or null
const at::Tensor *cuda_tensor(PyObject *o, at::ScalarType type)
{
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.scalar_type() == type && t.is_contiguous() ? &t : nullptr;
}

// did a conversion fail?  (binding.py's own then takes what it always took, or raises)
bool not_for_us()
{
    if (!PyErr_Occurred()) return false;
    PyErr_Clear();
    return true;
}

// the stream argument: an integer, or None for torch's current stream of `device`
bool stream_of(PyObject *o, c10::DeviceIndex device, void **stream)
{
    if (o == Py_None) {
        *stream = (void *)c10::cuda::getCurrentCUDAStream(device).stream();
        return true;
    }
    *stream = PyLong_AsVoidPtr(o);
    return *stream || !not_for_us();
}

// Where a call's memory comes from: the pool of the stream that it runs on.  What torch's current stream has given back may be
// in use by work that waits there, and a stream that was named does not wait for it.  Results are the caller's, who may give
// them back while its current stream still reads them.
class Memory {
  public:
    Memory(PyObject *stream_o, const at::Tensor &like, void *stream) : device_(like.device())
    {
        if (stream_o == Py_None) return;
        const auto current = c10::cuda::getCurrentCUDAStream(device_.index());
        if ((void *)current.stream() == stream) return;
        caller_ = current;
        named_ = c10::cuda::getStreamFromExternal((cudaStream_t)stream, device_.index());
    }
    at::Tensor result(at::IntArrayRef size, at::ScalarType type) const
    {
        return kept([&] { return at::detail::empty_cuda(size, type, device_, std::nullopt); });
    }
    at::Tensor result_strided(at::IntArrayRef size, at::IntArrayRef stride, at::ScalarType type) const
    {
        return kept([&] { return at::detail::empty_strided_cuda(size, stride, type, device_); });
    }
    at::Tensor workspace(int64_t bytes) const
    {
        const c10::cuda::OptionalCUDAStreamGuard guard(stream());
        return at::detail::empty_cuda({bytes}, at::kByte, device_, std::nullopt);
    }

  private:
    std::optional<c10::Stream> stream() const { return named_ ? std::optional<c10::Stream>(named_->unwrap()) : std::nullopt; }
    template <typename F>
    at::Tensor kept(F &&make) const
    {
        const c10::cuda::OptionalCUDAStreamGuard guard(stream());
        at::Tensor t = make();
        if (caller_ && t.numel()) c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), *caller_);
        return t;
    }
    const c10::Device device_;
    std::optional<c10::cuda::CUDAStream> named_, caller_;  // where they differ
};

template <typename F>
accerl_status without_gil(F &&call)
{
    accerl_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return st;
}

PyObject *wrapped(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

struct Names {
    PyObject *logits, *actions, *logp, *entropy, *value, *use_smaller, *stats, *kl, *grad;
} names;

void put(PyObject *dict, PyObject *key, at::Tensor t)
{
    PyObject *v = wrapped(std::move(t));
    PyDict_SetItem(dict, key, v);
    Py_XDECREF(v);
}

// what an observation batch and its uniforms have to be for the fast path
bool act_inputs(PyObject *u8, PyObject *obs_o, PyObject *u_o, const at::Tensor **obs, const at::Tensor **u, int64_t *b)
{
    *obs = cuda_tensor(obs_o, u8 == Py_True ? at::kByte : at::kFloat);
    *u = cuda_tensor(u_o, at::kFloat);
    if (!*obs || !*u || (*obs)->dim() < 1) return false;
    *b = (*obs)->size(0);
    return (*u)->numel() == *b && *b > 0 && *b <= INT32_MAX;
}

// act(handle, n_actions, frames, obs, uniforms, out, stream) -> (logits, actions, logp), or `out`
PyObject *py_act(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) return Py_BuildValue("");
    void *handle = PyLong_AsVoidPtr(a[0]);
    const int64_t A = PyLong_AsLongLong(a[1]);
    const at::Tensor *obs, *u;
    int64_t b;
    void *stream;
    if (not_for_us()) Py_RETURN_NONE;
    if (!act_inputs(a[2], a[3], a[4], &obs, &u, &b) || !stream_of(a[6], obs->device().index(), &stream)) Py_RETURN_NONE;
    const Memory memory(a[6], *obs, stream);
    void *dst[3];
    at::Tensor t[3];
    if (a[5] == Py_None) {
        t[0] = memory.result({b, A}, at::kFloat);
        t[1] = memory.result({b}, at::kInt);
        t[2] = memory.result({b}, at::kFloat);
        for (int i = 0; i < 3; ++i) dst[i] = t[i].data_ptr();
    } else {
        if (!PyTuple_Check(a[5]) || PyTuple_GET_SIZE(a[5]) != 3) Py_RETURN_NONE;
        for (int i = 0; i < 3; ++i) {
            PyObject *o = PyTuple_GET_ITEM(a[5], i);
            if (!THPVariable_Check(o)) Py_RETURN_NONE;
            dst[i] = THPVariable_Unpack(o).data_ptr();
        }
    }
    const void *obs_p = obs->data_ptr();
    const float *u_p = (const float *)u->data_ptr();
    const accerl_status st = without_gil([&] {
        return accerl_policy_act((accerl_policy *)handle, obs_p, u_p, (int32_t)b, (float *)dst[0], (int32_t *)dst[1],
                                 (float *)dst[2], stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    if (a[5] != Py_None) {
        Py_INCREF(a[5]);
        return a[5];
    }
    PyObject *r = PyTuple_New(3);
    if (!r) return nullptr;
    for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(r, i, wrapped(std::move(t[i])));
    return r;
}

// act_ex(handle, n_actions, frames, value_head, obs, uniforms, stream) -> dict
PyObject *py_act_ex(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) return Py_BuildValue("");
    void *handle = PyLong_AsVoidPtr(a[0]);
    const int64_t A = PyLong_AsLongLong(a[1]);
    const at::Tensor *obs, *u;
    int64_t b;
    void *stream;
    if (not_for_us()) Py_RETURN_NONE;
    if (!act_inputs(a[2], a[4], a[5], &obs, &u, &b) || !stream_of(a[6], obs->device().index(), &stream)) Py_RETURN_NONE;
    const Memory memory(a[6], *obs, stream);
    at::Tensor logits = memory.result({b, A}, at::kFloat), actions = memory.result({b}, at::kInt),
               logp = memory.result({b}, at::kFloat), entropy = memory.result({b}, at::kFloat), value;
    if (a[3] == Py_True) value = memory.result({b}, at::kFloat);
    const void *obs_p = obs->data_ptr();
    const float *u_p = (const float *)u->data_ptr();
    float *value_p = value.defined() ? (float *)value.data_ptr() : nullptr;
    const accerl_status st = without_gil([&] {
        return accerl_policy_act_ex((accerl_policy *)handle, obs_p, u_p, (int32_t)b, (float *)logits.data_ptr(),
                                    (int32_t *)actions.data_ptr(), (float *)logp.data_ptr(), value_p,
                                    (float *)entropy.data_ptr(), stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    PyObject *d = PyDict_New();
    if (!d) return nullptr;
    put(d, names.logits, std::move(logits));
    put(d, names.actions, std::move(actions));
    put(d, names.logp, std::move(logp));
    put(d, names.entropy, std::move(entropy));
    if (value.defined()) put(d, names.value, std::move(value));
    return d;
}

// act_mixed(smaller, original, n_actions, frames, value, obs, uniforms, select, alpha, stream) -> dict
PyObject *py_act_mixed(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 10) return Py_BuildValue("");
    void *smaller = PyLong_AsVoidPtr(a[0]), *original = PyLong_AsVoidPtr(a[1]);
    const int64_t A = PyLong_AsLongLong(a[2]);
    const double alpha = PyFloat_AsDouble(a[8]);
    const at::Tensor *obs, *u;
    int64_t b;
    void *stream;
    if (not_for_us()) Py_RETURN_NONE;
    const at::Tensor *select = cuda_tensor(a[7], at::kFloat);
    if (!act_inputs(a[3], a[5], a[6], &obs, &u, &b) || !select || select->numel() != b ||
        !stream_of(a[9], obs->device().index(), &stream))
        Py_RETURN_NONE;
    const Memory memory(a[9], *obs, stream);
    at::Tensor logits = memory.result({b, A}, at::kFloat), actions = memory.result({b}, at::kInt),
               logp = memory.result({b}, at::kFloat), entropy = memory.result({b}, at::kFloat),
               use = memory.result({b}, at::kByte), value;
    if (a[4] == Py_True) value = memory.result({b}, at::kFloat);
    const void *obs_p = obs->data_ptr();
    const float *u_p = (const float *)u->data_ptr(), *sel_p = (const float *)select->data_ptr();
    float *value_p = value.defined() ? (float *)value.data_ptr() : nullptr;
    const accerl_status st = without_gil([&] {
        return accerl_policy_act_mixed((accerl_policy *)smaller, (accerl_policy *)original, obs_p, u_p, sel_p,
                                       (float)alpha, (int32_t)b, (float *)logits.data_ptr(),
                                       (int32_t *)actions.data_ptr(), (float *)logp.data_ptr(), value_p,
                                       (float *)entropy.data_ptr(), (uint8_t *)use.data_ptr(), stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    PyObject *d = PyDict_New();
    if (!d) return nullptr;
    put(d, names.logits, std::move(logits));
    put(d, names.actions, std::move(actions));
    put(d, names.logp, std::move(logp));
    put(d, names.entropy, std::move(entropy));
    put(d, names.use_smaller, std::move(use));
    if (value.defined()) put(d, names.value, std::move(value));
    return d;
}

// kl(logits_original, logits_smaller, stream) -> (kl, mean_max)
PyObject *py_kl(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 3) return Py_BuildValue("");
    const at::Tensor *zo = cuda_tensor(a[0], at::kFloat), *zs = cuda_tensor(a[1], at::kFloat);
    void *stream;
    if (!zo || !zs || zo->dim() != 2 || zo->sizes() != zs->sizes() || zo->size(0) > INT32_MAX ||
        zo->size(1) > INT32_MAX || !stream_of(a[2], zo->device().index(), &stream))
        Py_RETURN_NONE;
    const Memory memory(a[2], *zo, stream);
    at::Tensor out = memory.result({zo->size(0)}, at::kFloat), stats = memory.result({2}, at::kFloat);
    const float *zo_p = (const float *)zo->data_ptr(), *zs_p = (const float *)zs->data_ptr();
    const int32_t b = (int32_t)zo->size(0), A = (int32_t)zo->size(1);
    const accerl_status st = without_gil([&] {
        return accerl_policy_kl(zo_p, zs_p, b, A, (float *)out.data_ptr(), (float *)stats.data_ptr(), stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrapped(std::move(out)), wrapped(std::move(stats)));
}

// vtrace(logp_smaller, logp_original, rewards, values, bootstrap, discounts, gamma, rho_hat, c_hat, stream)
// -> (vs, adv)
PyObject *py_vtrace(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 10) return Py_BuildValue("");
    const at::Tensor *in[6] = {};
    for (int i = 0; i < 6; ++i) {
        if (i == 5 && a[5] == Py_None) break;
        in[i] = cuda_tensor(a[i], at::kFloat);
        if (!in[i]) Py_RETURN_NONE;
        if (i == 4 ? in[4]->dim() != 1 || in[4]->size(0) != in[0]->size(1)
                   : in[i]->dim() != 2 || in[i]->sizes() != in[0]->sizes())
            Py_RETURN_NONE;
    }
    void *stream;
    if (in[0]->size(0) > INT32_MAX || in[0]->size(1) > INT32_MAX || !stream_of(a[9], in[0]->device().index(), &stream))
        Py_RETURN_NONE;
    const double gamma = PyFloat_AsDouble(a[6]), rho = PyFloat_AsDouble(a[7]), c = PyFloat_AsDouble(a[8]);
    if (not_for_us()) Py_RETURN_NONE;
    const Memory memory(a[9], *in[0], stream);
    at::Tensor vs = memory.result(in[0]->sizes(), at::kFloat), adv = memory.result(in[0]->sizes(), at::kFloat);
    const float *p[6];
    for (int i = 0; i < 6; ++i) p[i] = in[i] ? (const float *)in[i]->data_ptr() : nullptr;
    const int32_t steps = (int32_t)in[0]->size(0), b = (int32_t)in[0]->size(1);
    const accerl_status st = without_gil([&] {
        return accerl_vtrace(p[0], p[1], p[2], p[3], p[4], p[5], steps, b, (float)gamma, (float)rho, (float)c,
                             (float *)vs.data_ptr(), (float *)adv.data_ptr(), stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrapped(std::move(vs)), wrapped(std::move(adv)));
}

// ---- operators of the Learner's side ----------------------------------------------------------------------------

int dtype_code(at::ScalarType t)
{
    return t == at::kFloat ? ACCERL_F32 : t == at::kBFloat16 ? ACCERL_BF16 : t == at::kHalf ? ACCERL_F16 : -1;
}

// a CUDA matrix whose rows have adjacent elements
struct Rows {
    const at::Tensor *t = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    void *p = nullptr;
    int code = -1;  // accerl_dtype, or -1 for another type
};
bool rows_of(PyObject *o, Rows *r)
{
    if (!THPVariable_Check(o)) return false;
    r->t = &THPVariable_Unpack(o);
    if (!r->t->is_cuda() || r->t->dim() != 2) return false;
    r->rows = r->t->size(0);
    r->cols = r->t->size(1);
    if (r->rows < 1 || r->cols < 1 || r->rows > INT32_MAX || r->cols > INT32_MAX || (r->t->stride(1) != 1 && r->cols > 1)) return false;
    r->ld = r->rows > 1 ? r->t->stride(0) : std::max(r->cols, r->t->stride(0));
    if (r->ld < r->cols) return false;
    r->p = r->t->data_ptr();
    r->code = dtype_code(r->t->scalar_type());
    return true;
}
bool same_device(const at::Tensor &a, const at::Tensor &b) { return a.device() == b.device(); }

// a contiguous vector of n fp32 values on the device of `like`, or None where that is allowed
bool vector_of(PyObject *o, int64_t n, const at::Tensor &like, bool none, const float **p)
{
    *p = nullptr;
    if (o == Py_None) return none;
    const at::Tensor *t = cuda_tensor(o, at::kFloat);
    if (!t || t->dim() != 1 || t->size(0) != n || !same_device(*t, like)) return false;
    *p = (const float *)t->data_ptr();
    return true;
}

// q int8 and e uint8 of a checkpoint of rows x cols
bool ckpt_of(PyObject *o, int64_t rows, int64_t cols, const at::Tensor &like, Rows *q, Rows *e)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 2 || !rows_of(PyTuple_GET_ITEM(o, 0), q) || !rows_of(PyTuple_GET_ITEM(o, 1), e)) return false;
    const int64_t cols32 = (cols + 31) / 32 * 32;
    return q->t->scalar_type() == at::kChar && e->t->scalar_type() == at::kByte && q->rows == rows && e->rows == rows && q->cols >= cols32 &&
           e->cols >= cols32 / 32 && same_device(*q->t, like) && same_device(*e->t, like);
}

// q int8 and its scales as quant_rows makes them; the row distance as linear_i8 takes it
bool quantised_of(PyObject *qo, PyObject *so, const at::Tensor &like, Rows *q, const float **s)
{
    if (!rows_of(qo, q) || q->t->scalar_type() != at::kChar || !same_device(*q->t, like)) return false;
    if (q->rows == 1) q->ld = (q->ld + 15) / 16 * 16;
    return q->ld % 16 == 0 && ((uintptr_t)q->p & 15) == 0 && vector_of(so, q->rows, like, false, s);
}

template <typename F>
accerl_status on_device_of(const at::Tensor &t, F &&call)
{
    c10::cuda::CUDAGuard guard(t.device());
    return without_gil(call);
}

// quant_rows(x, stream) -> (q, scale)
PyObject *py_quant_rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Rows x;
    void *stream;
    if (n != 2 || !rows_of(a[0], &x) || x.code < 0 || !stream_of(a[1], x.t->device().index(), &stream)) Py_RETURN_NONE;
    const int64_t ld = (x.cols + 15) / 16 * 16;
    const Memory memory(a[1], *x.t, stream);
    at::Tensor q = memory.result({x.rows, ld}, at::kChar), scale = memory.result({x.rows}, at::kFloat);
    const accerl_status st = on_device_of(*x.t, [&] {
        return accerl_quant_rows(x.p, x.ld, x.code, x.rows, (int32_t)x.cols, (int8_t *)q.data_ptr(), ld, (float *)scale.data_ptr(), stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    return Py_BuildValue("(NN)", wrapped(ld == x.cols ? q : q.narrow(1, 0, x.cols)), wrapped(std::move(scale)));
}

// linear_i8(x, wq, w_scale, bias, relu, out_dtype or None, stream) -> y
PyObject *py_linear_i8(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Rows x, w;
    accerl_linear_i8_args g = {};
    void *stream;
    if (n != 7 || !rows_of(a[0], &x) || x.code < 0 || !quantised_of(a[1], a[2], *x.t, &w, &g.w_scale) || w.cols != x.cols ||
        !vector_of(a[3], w.rows, *x.t, true, &g.bias) || !stream_of(a[6], x.t->device().index(), &stream))
        Py_RETURN_NONE;
    const int relu = PyObject_IsTrue(a[4]);
    if (relu < 0) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    at::ScalarType type = x.t->scalar_type();
    if (a[5] != Py_None) {
        if (!THPDtype_Check(a[5])) Py_RETURN_NONE;
        type = reinterpret_cast<THPDtype *>(a[5])->scalar_type;
    }
    if (dtype_code(type) < 0) Py_RETURN_NONE;
    const Memory memory(a[6], *x.t, stream);
    at::Tensor y = memory.result({x.rows, w.rows}, type), space;
    g.workspace_bytes = accerl_linear_i8_workspace((int32_t)x.rows, (int32_t)x.cols, x.code);
    if (g.workspace_bytes) {
        space = memory.workspace(g.workspace_bytes);
        g.workspace = space.data_ptr();
    }
    g.x = x.p;
    g.w = (const int8_t *)w.p;
    g.y = y.data_ptr();
    g.ld_x = x.ld;
    g.ld_w = w.ld;
    g.ld_y = w.rows;
    g.tokens = (int32_t)x.rows;
    g.n = (int32_t)w.rows;
    g.k = (int32_t)x.cols;
    g.x_dtype = x.code;
    g.y_dtype = dtype_code(type);
    g.relu = relu;
    const accerl_status st = on_device_of(*x.t, [&] { return accerl_linear_i8(&g, stream); });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    return wrapped(std::move(y));
}

// ckpt_save(x, act code, stream) -> (y, (q, e)); y is x without an activation
PyObject *py_ckpt_save(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Rows x;
    void *stream;
    if (n != 3 || !rows_of(a[0], &x) || x.code < 0 || !stream_of(a[2], x.t->device().index(), &stream)) Py_RETURN_NONE;
    const long act = PyLong_AsLong(a[1]);
    if (not_for_us()) Py_RETURN_NONE;
    const int64_t cols32 = (x.cols + 31) / 32 * 32;
    const Memory memory(a[2], *x.t, stream);
    at::Tensor q = memory.result({x.rows, cols32}, at::kChar), e = memory.result({x.rows, cols32 / 32}, at::kByte), y;
    if (act != ACCERL_ACT_NONE) y = memory.result({x.rows, x.cols}, x.t->scalar_type());
    const accerl_status st = on_device_of(*x.t, [&] {
        return accerl_ckpt_save(x.p, x.ld, x.code, x.rows, (int32_t)x.cols, (int32_t)act, y.defined() ? y.data_ptr() : nullptr, x.cols,
                                (int8_t *)q.data_ptr(), cols32, (uint8_t *)e.data_ptr(), cols32 / 32, stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    PyObject *yo = a[0];
    if (y.defined()) yo = wrapped(std::move(y));
    else Py_INCREF(yo);
    return Py_BuildValue("(N(NN))", yo, wrapped(std::move(q)), wrapped(std::move(e)));
}

// ckpt_load(ckpt, cols, dtype, stream) -> x
PyObject *py_ckpt_load(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 4 || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 2 || !THPDtype_Check(a[2])) Py_RETURN_NONE;
    const at::ScalarType type = reinterpret_cast<THPDtype *>(a[2])->scalar_type;
    const int64_t cols = PyLong_AsLongLong(a[1]);
    Rows q, e, like;
    void *stream;
    if (not_for_us() || cols < 1 || cols > INT32_MAX || dtype_code(type) < 0 || !rows_of(PyTuple_GET_ITEM(a[0], 0), &like) ||
        !ckpt_of(a[0], like.rows, cols, *like.t, &q, &e) || !stream_of(a[3], like.t->device().index(), &stream))
        Py_RETURN_NONE;
    const Memory memory(a[3], *q.t, stream);
    at::Tensor x = memory.result({q.rows, cols}, type);
    const accerl_status st = on_device_of(*q.t, [&] {
        return accerl_ckpt_load((const int8_t *)q.p, q.ld, (const uint8_t *)e.p, e.ld, q.rows, (int32_t)cols, x.data_ptr(), cols,
                                dtype_code(type), stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    return wrapped(std::move(x));
}

// ckpt_act_backward(dy, ckpt, act code, stream) -> dx
PyObject *py_ckpt_act_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Rows dy, q, e;
    void *stream;
    if (n != 4 || !rows_of(a[0], &dy) || dy.code < 0 || !ckpt_of(a[1], dy.rows, dy.cols, *dy.t, &q, &e) ||
        !stream_of(a[3], dy.t->device().index(), &stream))
        Py_RETURN_NONE;
    const long act = PyLong_AsLong(a[2]);
    if (not_for_us()) Py_RETURN_NONE;
    const Memory memory(a[3], *dy.t, stream);
    at::Tensor dx = memory.result({dy.rows, dy.cols}, dy.t->scalar_type());
    const accerl_status st = on_device_of(*dy.t, [&] {
        return accerl_ckpt_act_backward(dy.p, dy.ld, dy.code, (const int8_t *)q.p, q.ld, (const uint8_t *)e.p, e.ld, dy.rows, (int32_t)dy.cols,
                                        (int32_t)act, dx.data_ptr(), dy.cols, stream);
    });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    return wrapped(std::move(dx));
}

// ckpt_weight_grad(dy, ckpt, cols, out_dtype or None, bias, stream) -> (dw, db or None)
PyObject *py_ckpt_weight_grad(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Rows dy, q, e;
    void *stream;
    if (n != 6 || !rows_of(a[0], &dy) || dy.code < 0) Py_RETURN_NONE;
    const int64_t k = PyLong_AsLongLong(a[2]);
    if (not_for_us() || k < 1 || k > INT32_MAX || !ckpt_of(a[1], dy.rows, k, *dy.t, &q, &e) ||
        !stream_of(a[5], dy.t->device().index(), &stream))
        Py_RETURN_NONE;
    at::ScalarType type = dy.t->scalar_type();
    if (a[3] != Py_None) {
        if (!THPDtype_Check(a[3])) Py_RETURN_NONE;
        type = reinterpret_cast<THPDtype *>(a[3])->scalar_type;
    }
    const int bias = PyObject_IsTrue(a[4]);
    if (bias < 0) PyErr_Clear();
    if (bias < 0 || dtype_code(type) < 0) Py_RETURN_NONE;
    const Memory memory(a[5], *dy.t, stream);
    at::Tensor dw = memory.result({dy.cols, k}, type), db, space;
    if (bias) db = memory.result({dy.cols}, type);
    accerl_weight_grad_args g = {};
    g.dy = dy.p;
    g.q = (const int8_t *)q.p;
    g.e = (const uint8_t *)e.p;
    g.dw = dw.data_ptr();
    g.db = bias ? db.data_ptr() : nullptr;
    g.ld_dy = dy.ld;
    g.ld_q = q.ld;
    g.ld_e = e.ld;
    g.ld_dw = k;
    g.tokens = (int32_t)dy.rows;
    g.n = (int32_t)dy.cols;
    g.k = (int32_t)k;
    g.dy_dtype = dy.code;
    g.out_dtype = dtype_code(type);
    g.workspace_bytes = accerl_ckpt_weight_grad_workspace(&g);
    if (g.workspace_bytes) {
        space = memory.workspace(g.workspace_bytes);
        g.workspace = space.data_ptr();
    }
    const accerl_status st = on_device_of(*dy.t, [&] { return accerl_ckpt_weight_grad(&g, stream); });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    PyObject *dbo = Py_None;
    if (bias) dbo = wrapped(std::move(db));
    else Py_INCREF(dbo);
    return Py_BuildValue("(NN)", wrapped(std::move(dw)), dbo);
}

// policy_loss(logits, actions, logp_old, advantages, weights, logits_ref, logp_ref, clip_low, clip_high, kl_coef,
// entropy_coef, grad (True, False or a tensor), stream) -> dict
PyObject *py_policy_loss(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    Rows z, zr, gr;
    accerl_policy_loss_args g = {};
    void *stream;
    if (n != 13 || !rows_of(a[0], &z) || z.code < 0 || !THPVariable_Check(a[1])) Py_RETURN_NONE;
    const at::Tensor &like = *z.t, &actions = THPVariable_Unpack(a[1]);
    const bool wide = actions.scalar_type() == at::kLong;
    if (!actions.is_cuda() || !same_device(actions, like) || actions.dim() != 1 || actions.size(0) != z.rows || !actions.is_contiguous() ||
        (!wide && actions.scalar_type() != at::kInt) || !vector_of(a[2], z.rows, like, false, &g.logp_old) ||
        !vector_of(a[3], z.rows, like, false, &g.advantages) || !vector_of(a[4], z.rows, like, true, &g.weights) ||
        !vector_of(a[6], z.rows, like, true, &g.logp_ref) || !stream_of(a[12], like.device().index(), &stream))
        Py_RETURN_NONE;
    if (a[5] != Py_None && (!rows_of(a[5], &zr) || zr.code != z.code || zr.rows != z.rows || zr.cols != z.cols || !same_device(*zr.t, like)))
        Py_RETURN_NONE;
    const double c[4] = {PyFloat_AsDouble(a[7]), PyFloat_AsDouble(a[8]), PyFloat_AsDouble(a[9]), PyFloat_AsDouble(a[10])};
    if (not_for_us()) Py_RETURN_NONE;
    const Memory memory(a[12], like, stream);
    at::Tensor grad;
    if (a[11] == Py_True) {
        // rows as far apart as the logits', which then lie alike to 16 bytes; but not those of the last token of sequences
        g.ld_grad = z.ld < 2 * z.cols ? z.ld : (z.cols + 7) / 8 * 8;
        grad = memory.result_strided({z.rows, z.cols}, {g.ld_grad, 1}, like.scalar_type());
        g.grad = grad.data_ptr();
    } else if (a[11] != Py_False) {
        if (!rows_of(a[11], &gr) || gr.code != z.code || gr.rows != z.rows || gr.cols != z.cols || !same_device(*gr.t, like)) Py_RETURN_NONE;
        g.grad = gr.p;
        g.ld_grad = gr.ld;
    }
    const int64_t t = z.rows;
    at::Tensor f = memory.result({8 + 5 * t}, at::kFloat);
    float *fp = (float *)f.data_ptr();
    g.logits = z.p;
    g.logits_ref = zr.p;
    g.actions = actions.data_ptr();
    g.ld_logits = z.ld;
    g.ld_logits_ref = zr.ld;
    g.rows = (int32_t)t;
    g.n_actions = (int32_t)z.cols;
    g.dtype = z.code;
    g.actions64 = wide;
    g.clip_low = (float)c[0];
    g.clip_high = (float)c[1];
    g.kl_coef = (float)c[2];
    g.entropy_coef = (float)c[3];
    g.stats = fp;
    g.terms = fp + 8;
    g.logp = fp + 8 + 2 * t;
    g.kl = fp + 8 + 3 * t;
    g.entropy = fp + 8 + 4 * t;
    const accerl_status st = on_device_of(like, [&] { return accerl_policy_loss(&g, stream); });
    if (st != ACCERL_OK) return PyLong_FromLong(st);
    PyObject *d = PyDict_New();
    if (!d) return nullptr;
    put(d, names.stats, f.narrow(0, 0, 8));
    put(d, names.logp, f.narrow(0, 8 + 2 * t, t));
    put(d, names.kl, f.narrow(0, 8 + 3 * t, t));
    put(d, names.entropy, f.narrow(0, 8 + 4 * t, t));
    if (grad.defined()) put(d, names.grad, std::move(grad));
    else PyDict_SetItem(d, names.grad, a[11] == Py_False ? Py_None : a[11]);
    return d;
}

// act_noalloc(handle, obs, uniforms, batch, logits, actions, logp, stream): raw addresses -> status, or None for
// arguments that are no plain integers (ctypes pointers, numpy integers: binding.py passes those through ctypes)
PyObject *py_act_noalloc(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 8) return Py_BuildValue("");
    void *p[8] = {};
    for (int i = 0; i < 8; ++i) {
        if (i == 3 || a[i] == Py_None) continue;
        if (!PyLong_Check(a[i])) Py_RETURN_NONE;
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i] && not_for_us()) Py_RETURN_NONE;
    }
    if (!PyLong_Check(a[3])) Py_RETURN_NONE;
    const long batch = PyLong_AsLong(a[3]);
    if (batch == -1 && not_for_us()) Py_RETURN_NONE;
    const accerl_status st = without_gil([&] {
        return accerl_policy_act_noalloc((accerl_policy *)p[0], p[1], (const float *)p[2], (int32_t)batch, (float *)p[4],
                                         (int32_t *)p[5], (float *)p[6], p[7]);
    });
    return PyLong_FromLong(st);
}

// C++ exceptions (a failed allocation among them) become the Python exceptions torch raises for them
template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    return F(self, a, n);
    END_HANDLE_TH_ERRORS
}

#define FAST(f) (PyCFunction)(void (*)(void))guarded<f>, METH_FASTCALL
PyMethodDef methods[] = {{"act", FAST(py_act), nullptr},
                         {"act_ex", FAST(py_act_ex), nullptr},
                         {"act_mixed", FAST(py_act_mixed), nullptr},
                         {"act_noalloc", FAST(py_act_noalloc), nullptr},
                         {"ckpt_act_backward", FAST(py_ckpt_act_backward), nullptr},
                         {"ckpt_load", FAST(py_ckpt_load), nullptr},
                         {"ckpt_save", FAST(py_ckpt_save), nullptr},
                         {"ckpt_weight_grad", FAST(py_ckpt_weight_grad), nullptr},
                         {"kl", FAST(py_kl), nullptr},
                         {"linear_i8", FAST(py_linear_i8), nullptr},
                         {"policy_loss", FAST(py_policy_loss), nullptr},
                         {"quant_rows", FAST(py_quant_rows), nullptr},
                         {"vtrace", FAST(py_vtrace), nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void)
{
    names.logits = PyUnicode_InternFromString("logits");
    names.actions = PyUnicode_InternFromString("actions");
    names.logp = PyUnicode_InternFromString("logp");
    names.entropy = PyUnicode_InternFromString("entropy");
    names.value = PyUnicode_InternFromString("value");
    names.use_smaller = PyUnicode_InternFromString("use_smaller");
    names.stats = PyUnicode_InternFromString("stats");
    names.kl = PyUnicode_InternFromString("kl");
    names.grad = PyUnicode_InternFromString("grad");
    return PyModule_Create(&module);
}
