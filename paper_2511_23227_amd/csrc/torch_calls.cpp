// The Python side of the operators around the convolution in compiled code: checks of torch tensors, outputs, and the calls of libpcpp.so.
// binding.py's functions of the same names wrap the results.
//
// Their smallest calls take the GPU 3 us, so what the host does is what they cost: block_norm_fwd of three rows took 10.5 us through ctypes, of which
// the launch is 3.3, and takes 5.8 so; block_norm_bwd 21.8 and 12, pack and unpack 14.5 and 10.4, log_probs_fwd of a split row 18.4 and 11.4.
//
// Every function returns its outputs as a tuple, or the status of the call where it is not PCPP_OK.  Tensors that do not fit raise
// AssertionError, types TypeError.
#include <Python.h>

#include <dlfcn.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pcpp.h"

namespace {

using at::Tensor;

struct Fail {
    PyObject *type;
    const char *what;
};
inline void need(bool ok, const char *what)
{
    if (!ok) throw Fail{PyExc_AssertionError, what};
}

// ---- the library's functions, by the handle that ctypes opened it with ------------------------------------------------------------
struct {
#define CALL(name) decltype(&pcpp_##name) name
    CALL(act_pack);
    CALL(act_unpack);
    CALL(mvmr_packed_workspace_bytes);
    CALL(mvmr_bwd_weight_packed);
    CALL(block_norm_fwd);
    CALL(block_norm_workspace_bytes);
    CALL(block_norm_bwd);
    CALL(log_probs_workspace_bytes);
    CALL(log_probs_fwd);
    CALL(log_probs_bwd);
    CALL(dropout_fwd);
    CALL(dropout_bwd);
    CALL(group_norm_workspace_bytes);
    CALL(group_norm_fwd);
    CALL(group_norm_bwd);
    CALL(mx_pack);
    CALL(mx_unpack);
    CALL(mx_product_workspace_bytes);
    CALL(mx_product);
    CALL(mx_linear_workspace_bytes);
    CALL(mx_linear);
#undef CALL
} lib;

// ---- arguments ---------------------------------------------------------------------------------------------------------------
struct Args {
    PyObject *const *a;
    Py_ssize_t n, at = 0;
    int64_t device = -1;                                          // of the tensors so far
    PyObject *next()
    {
        if (at >= n) throw Fail{PyExc_TypeError, "too few arguments"};
        return a[at++];
    }
    const Tensor *optional()
    {
        PyObject *o = next();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) throw Fail{PyExc_TypeError, "expected a tensor"};
        const Tensor &t = THPVariable_Unpack(o);
        need(t.is_cuda(), "tensors must be on the GPU");
        need(device < 0 || device == t.get_device(), "tensors must be on one GPU");
        device = t.get_device();
        return &t;
    }
    const Tensor &tensor()
    {
        const Tensor *t = optional();
        if (!t) throw Fail{PyExc_TypeError, "expected a tensor"};
        return *t;
    }
    int64_t integer()
    {
        const long long v = PyLong_AsLongLong(next());
        if (v == -1 && PyErr_Occurred()) throw Fail{nullptr, nullptr};
        return v;
    }
    int small()
    {
        const int64_t v = integer();
        if (v != (int)v) throw Fail{PyExc_OverflowError, "argument out of range"};
        return (int)v;
    }
    float number()
    {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw Fail{nullptr, nullptr};
        return (float)v;
    }
    // the last two arguments: the current device and its stream
    void *stream()
    {
        need(integer() == device, "tensors must be on the current device");
        void *p = PyLong_AsVoidPtr(next());
        if (!p && PyErr_Occurred()) throw Fail{nullptr, nullptr};
        return p;
    }
};

int code_of(at::ScalarType t)
{
    if (t == at::kFloat) return PCPP_F32;
    if (t == at::kBFloat16) return PCPP_BF16;
    throw Fail{PyExc_TypeError, "unsupported dtype (float32 and bfloat16 are)"};
}
at::ScalarType type_of(int64_t code)
{
    if (code != PCPP_F32 && code != PCPP_BF16) throw Fail{PyExc_TypeError, "unsupported dtype (float32 and bfloat16 are)"};
    return code == PCPP_F32 ? at::kFloat : at::kBFloat16;
}
int code_bytes(int64_t c) { return (int)((c + 127) / 128 * 4); }

bool shape(const Tensor &t, int64_t n, int64_t c) { return t.dim() == 2 && t.size(0) == n && t.size(1) == c; }
void need_rows(const Tensor &t, int64_t n, int64_t c, const char *what) { need(shape(t, n, c) && t.is_contiguous(), what); }
int channels(const Tensor &t)
{
    need(t.size(1) <= INT32_MAX, "too many channels");
    return (int)t.size(1);
}

// Row pitch of a [n, c] tensor whose rows are contiguous, in elements.
int64_t pitch(const Tensor &t)
{
    const int64_t n = t.size(0), c = t.size(1);
    need(c <= 1 || t.stride(1) == 1, "the channels of a row must lie side by side");
    if (n <= 1) return c;
    need(t.stride(0) >= c, "rows must not overlap");
    return t.stride(0);
}

struct Rows8 {
    const Tensor *q = nullptr, *codes = nullptr;
    int8_t *at() const { return q ? static_cast<int8_t *>(q->data_ptr()) : nullptr; }
    uint8_t *codes_at() const { return codes ? static_cast<uint8_t *>(codes->data_ptr()) : nullptr; }
};
Rows8 rows8(const Tensor *q, const Tensor *codes)
{
    if (!q && !codes) return Rows8{};
    need(q && codes, "q and codes belong together");
    need(q->scalar_type() == at::kChar && codes->scalar_type() == at::kByte, "q is int8 and codes uint8");
    need(q->dim() == 2 && q->is_contiguous() && codes->is_contiguous() && shape(*codes, q->size(0), code_bytes(q->size(1))),
         "q is [n, c] and codes [n, pcpp_act_code_bytes(c)], both contiguous");
    return Rows8{q, codes};
}

const float *weights(const Tensor *w, int64_t c)
{
    if (!w) return nullptr;
    need(w->scalar_type() == at::kFloat && w->dim() == 1 && w->size(0) == c && w->is_contiguous(), "weights are float32 [c]");
    return static_cast<const float *>(w->data_ptr());
}
const void *at_of(const Tensor *t) { return t ? t->data_ptr() : nullptr; }

// Every output has a storage of its own, at 0.6 us each: tensors of different types in one cannot be saved, and one that is kept or saved would
// hold them all.
Tensor empty(at::IntArrayRef size, at::ScalarType type, const Tensor &like) { return at::empty(size, like.options().dtype(type).requires_grad(false)); }
// The caller's workspace, or a new one where it is too small or does not lie in one piece (an expanded tensor's nbytes() are not there).
Tensor workspace_of(size_t bytes, const Tensor *given, const Tensor &like)
{
    if (given && given->is_contiguous() && (size_t)given->nbytes() >= bytes) return *given;
    return empty({(int64_t)(bytes > 256 ? bytes : 256)}, at::kByte, like);
}

// new rows in 8 bits: q and codes
std::pair<Tensor, Tensor> new_rows8(int64_t n, int64_t c, const Tensor &like)
{
    return {empty({n, c}, at::kChar, like), empty({n, code_bytes(c)}, at::kByte, like)};
}

// A tensor of the caller's that a call has written: autograd is to refuse to go on with what it saved of it.
void written(const Tensor *t)
{
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// ---- results ------------------------------------------------------------------------------------------------------------------
PyObject *wrapped(const Tensor &t)
{
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
template <typename... T> PyObject *result(int rc, const T &...t)
{
    if (rc != PCPP_OK) return PyLong_FromLong(rc);
    PyObject *tuple = PyTuple_New(sizeof...(T));
    if (!tuple) return nullptr;
    Py_ssize_t i = 0;
    bool ok = true;
    auto put = [&](PyObject *o) {
        ok = ok && o;
        PyTuple_SET_ITEM(tuple, i++, o);
    };
    (put(wrapped(t)), ...);
    if (ok) return tuple;
    Py_DECREF(tuple);
    return nullptr;
}
// no C++ exception leaves a function
template <typename F> PyObject *guarded(PyObject *const *a, Py_ssize_t n, F f)
{
    try {
        Args args{a, n};
        return f(args);
    } catch (const Fail &e) {
        if (e.type) PyErr_SetString(e.type, e.what);
    } catch (const std::bad_alloc &) {
        PyErr_NoMemory();
    } catch (const python_error &) {                   // (raised by torch, set already)
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

// ---- the calls ----------------------------------------------------------------------------------------------------------------
// (x, q or None, codes or None, device, stream) -> (q, codes)
PyObject *act_pack(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const Tensor *q = args.optional(), *codes = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2 && x.is_contiguous(), "x is [n, c], contiguous");
        const int64_t n = x.size(0);
        const int c = channels(x), code = code_of(x.scalar_type());
        const Rows8 given = rows8(q, codes);
        if (given.q) need(shape(*given.q, n, c), "q has another shape than x");
        const auto [to, to_codes] = given.q ? std::pair<Tensor, Tensor>(*given.q, *given.codes) : new_rows8(n, c, x);
        const int rc = lib.act_pack(x.data_ptr(), code, n, c, static_cast<int8_t *>(to.data_ptr()), static_cast<uint8_t *>(to_codes.data_ptr()), stream);
        written(given.q);
        written(given.codes);
        return result(rc, to, to_codes);
    });
}

// (q, codes, dtype code, out or None, device, stream) -> (x,)
PyObject *act_unpack(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &q = args.tensor(), &codes = args.tensor();
        const int64_t code = args.integer();
        const Tensor *given = args.optional();
        void *stream = args.stream();
        const Rows8 rows = rows8(&q, &codes);
        const int64_t n = q.size(0);
        const int c = channels(q);
        if (given) need_rows(*given, n, c, "out has another shape than q, or is not contiguous");
        const Tensor out = given ? *given : empty({n, c}, type_of(code), q);
        const int rc = lib.act_unpack(rows.at(), rows.codes_at(), n, c, out.data_ptr(), code_of(out.scalar_type()), stream);
        written(given);
        return result(rc, out);
    });
}

// (q, codes, dy, tri_o, tri_i, tri_k, seg_offsets, plan or None, plan_flags, n_triplets, n_in, n_out, K, dw or None, workspace or None,
//  device, stream) -> (dw,)
PyObject *weight_packed(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &q = args.tensor(), &codes = args.tensor(), &dy = args.tensor();
        const Tensor &tri_o = args.tensor(), &tri_i = args.tensor(), &tri_k = args.tensor(), &seg = args.tensor();
        const Tensor *plan = args.optional();
        const int flags = args.small();
        const int64_t n = args.integer(), n_in = args.integer(), n_out = args.integer();
        const int K = args.small();
        const Tensor *given = args.optional(), *workspace = args.optional();
        void *stream = args.stream();
        const Rows8 x = rows8(&q, &codes);
        need(q.size(0) == n_in && dy.dim() == 2 && dy.size(0) == n_out && dy.is_contiguous(), "rows of x and dy are the triplets' inputs and outputs");
        for (const Tensor *t : {&tri_o, &tri_i, &tri_k})
            need(t->scalar_type() == at::kInt && t->is_contiguous() && t->numel() >= n, "triplets are int32 [n_triplets]");
        need(seg.scalar_type() == at::kLong && seg.is_contiguous() && seg.numel() > K, "seg_offsets are int64 [K + 1]");
        need(!plan || plan->is_contiguous(), "the plan must be contiguous");
        const int c_in = channels(q), c_out = channels(dy), code = code_of(dy.scalar_type());
        if (given)
            need(given->scalar_type() == at::kFloat && given->is_contiguous() && given->dim() == 3 && given->size(0) == K && given->size(1) == c_out &&
                     given->size(2) == c_in, "dw is float32 [K, c_out, c_in], contiguous");
        const Tensor dw = given ? *given : empty({K, c_out, c_in}, at::kFloat, dy);
        const Tensor ws = workspace_of(lib.mvmr_packed_workspace_bytes(n_in, n_out, n, c_in, c_out, K, code), workspace, dy);
        auto words = [](const Tensor &t) { return static_cast<const int32_t *>(t.data_ptr()); };
        const int rc = lib.mvmr_bwd_weight_packed(x.at(), x.codes_at(), dy.data_ptr(), static_cast<float *>(dw.data_ptr()), code, n_in, n_out, c_in, c_out, K,
                                                  words(tri_o), words(tri_i), words(tri_k), static_cast<const int64_t *>(seg.data_ptr()), n, at_of(plan),
                                                  plan ? plan->nbytes() : 0, flags, ws.data_ptr(), ws.nbytes(), stream);
        written(given);
        return result(rc, dw);
    });
}

struct Gate {
    const void *at = nullptr;
    int64_t ld = 0;
    int cols = 0;
    Gate(const Tensor *t, int64_t n, int64_t c, at::ScalarType type)
    {
        if (!t) return;
        need(t->scalar_type() == type && t->dim() == 2 && t->size(0) == n && (t->size(1) == c || t->size(1) == 1), "the gate is [n, c] or [n, 1], of the block's type");
        at = t->data_ptr();
        ld = pitch(*t);
        cols = (int)t->size(1);
    }
};

// (x, f, gate, w_post, w_pre, post, pre, residual_scale, eps, dtype code (-1: x's), pack_f, pack_h, device, stream) -> (r, h, fq, fcodes, hq, hcodes)
PyObject *block_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const Tensor *f = args.optional(), *gate = args.optional(), *w_post = args.optional(), *w_pre = args.optional();
        const int post = args.small(), pre = args.small();
        const float scale = args.number(), eps = args.number();
        const int64_t wanted = args.integer();
        const bool pack_f = args.integer(), pack_h = args.integer();
        void *stream = args.stream();
        need(x.dim() == 2 && x.is_contiguous(), "x is [n, c], contiguous");
        const int64_t n = x.size(0);
        const int c = channels(x);
        if (f) need(shape(*f, n, c), "f has another shape than x");
        const at::ScalarType type = f ? f->scalar_type() : (wanted < 0 ? x.scalar_type() : type_of(wanted));
        const int stream_code = code_of(x.scalar_type()), code = code_of(type);
        const Gate g(gate, n, c, type);
        Tensor r, h, fq, fe, hq, he;
        if (f) r = empty({n, c}, x.scalar_type(), x);
        if (pre != PCPP_NORM_NONE) h = empty({n, c}, type, x);
        if (pack_f) std::tie(fq, fe) = new_rows8(n, c, x);
        if (pack_h) std::tie(hq, he) = new_rows8(n, c, x);
        auto to = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        const int rc = lib.block_norm_fwd(x.data_ptr(), at_of(f), f ? pitch(*f) : c, g.at, g.ld, g.cols, weights(w_post, c), weights(w_pre, c), post, pre, scale,
                                          eps, n, c, stream_code, code, to(r), to(h), static_cast<int8_t *>(to(fq)), static_cast<uint8_t *>(to(fe)),
                                          static_cast<int8_t *>(to(hq)), static_cast<uint8_t *>(to(he)), stream);
        return result(rc, r, h, fq, fe, hq, he);
    });
}

// (dr, dh, r, f, fq, fcodes, gate, w_post, w_pre, post, pre, residual_scale, eps, dtype code (-1: of dh, f, gate, the stream), block, workspace,
//  device, stream) -> (dx, df, dgate, dw_post, dw_pre)
PyObject *block_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor *dr = args.optional(), *dh = args.optional(), *r = args.optional(), *f = args.optional();
        const Tensor *fq = args.optional(), *fe = args.optional(), *gate = args.optional(), *w_post = args.optional(), *w_pre = args.optional();
        const int post = args.small(), pre = args.small();
        const float scale = args.number(), eps = args.number();
        const int64_t wanted = args.integer();
        const bool block = args.integer();
        const Tensor *workspace = args.optional();
        void *stream = args.stream();
        const Tensor *some = dr ? dr : dh;
        need(some, "neither dr nor dh");
        need(some->dim() == 2, "gradients are [n, c]");
        const int64_t n = some->size(0);
        const int c = channels(*some);
        for (const Tensor *t : {dr, dh, r})
            if (t) need_rows(*t, n, c, "dr, dh and r are [n, c], contiguous");
        const Rows8 f8 = rows8(fq, fe);
        if (f8.q) need(shape(*f8.q, n, c), "f has another shape than the gradients");
        if (f) need(shape(*f, n, c), "f has another shape than the gradients");
        need(r || dr, "neither dr nor r says the stream's type");
        const at::ScalarType stream_type = r ? r->scalar_type() : dr->scalar_type();
        need(!dr || dr->scalar_type() == stream_type, "dr and r are of the stream's type");
        const at::ScalarType type = dh ? dh->scalar_type() : f ? f->scalar_type() : gate ? gate->scalar_type() : wanted >= 0 ? type_of(wanted) : stream_type;
        need(!f || f->scalar_type() == type, "f is of the block's type");
        const int stream_code = code_of(stream_type), code = code_of(type);
        const Gate g(gate, n, c, type);
        Tensor dx = empty({n, c}, stream_type, *some), df, dgate, dw_post, dw_pre;
        if (block) df = empty({n, c}, type, *some);
        if (gate) dgate = empty({n, g.cols}, type, *some);
        const bool of_post = block && (f || f8.q) && (post != PCPP_NORM_NONE || w_post), of_pre = pre != PCPP_NORM_NONE;
        if (of_post) dw_post = empty({c}, at::kFloat, *some);
        if (of_pre) dw_pre = empty({c}, at::kFloat, *some);
        const Tensor ws = workspace_of(lib.block_norm_workspace_bytes(n, c), workspace, *some);
        auto to = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        const int rc = lib.block_norm_bwd(at_of(dr), at_of(dh), at_of(r), at_of(f), f ? pitch(*f) : c, f8.at(), f8.codes_at(), g.at, g.ld, g.cols,
                                          weights(w_post, c), weights(w_pre, c), post, pre, scale, eps, n, c, stream_code, code, dx.data_ptr(), to(df), to(dgate),
                                          static_cast<float *>(to(dw_post)), static_cast<float *>(to(dw_pre)), ws.data_ptr(), ws.nbytes(), stream);
        return result(rc, dx, df, dgate, dw_post, dw_pre);
    });
}

const int32_t *labels_at(const Tensor *t, int64_t n)
{
    if (!t) return nullptr;
    need(t->scalar_type() == at::kInt && t->dim() == 1 && t->size(0) == n && t->is_contiguous(), "labels are int32 [n]");
    return static_cast<const int32_t *>(t->data_ptr());
}
const float *floats_at(const Tensor *t, int64_t n)
{
    if (!t) return nullptr;
    need(t->scalar_type() == at::kFloat && t->dim() == 1 && t->size(0) == n && t->is_contiguous(), "float32 [n] is wanted");
    return static_cast<const float *>(t->data_ptr());
}

// (logits, labels, n_top, workspace, device, stream) -> (log_prob, entropy, max_log_sum, top_log_prob, top_index)
PyObject *log_probs_fwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const Tensor *labels = args.optional();
        const int n_top = args.small();
        const Tensor *workspace = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2, "logits are [n, v]");
        const int64_t n = x.size(0), v = x.size(1), ld = pitch(x);
        const int32_t *label_at = labels_at(labels, n);
        const int code = code_of(x.scalar_type());
        const int64_t k = n_top > 0 && n_top <= PCPP_MAX_ALTERNATIVES ? n_top : 0;       // (others are refused by the call)
        Tensor log_prob, top, index;
        const Tensor stats = empty({n, 2}, at::kFloat, x), entropy = empty({n}, at::kFloat, x);
        if (labels) log_prob = empty({n}, at::kFloat, x);
        if (k) top = empty({n, k}, at::kFloat, x), index = empty({n, k}, at::kInt, x);
        const size_t bytes = lib.log_probs_workspace_bytes(n, v, n_top);
        Tensor ws;
        if (bytes) ws = workspace_of(bytes, workspace, x);
        auto to = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        const int rc = lib.log_probs_fwd(x.data_ptr(), code, n, v, ld, label_at, n_top, static_cast<float *>(to(log_prob)), static_cast<float *>(entropy.data_ptr()),
                                         static_cast<float *>(stats.data_ptr()), static_cast<float *>(to(top)), static_cast<int32_t *>(to(index)), to(ws),
                                         bytes ? ws.nbytes() : 0, stream);
        return result(rc, log_prob, entropy, stats, top, index);
    });
}

// (logits, labels, max_log_sum, entropy, d_log_prob, d_entropy, out, device, stream) -> (d_logits,)
PyObject *log_probs_bwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const Tensor *labels = args.optional();
        const Tensor &stats = args.tensor();
        const Tensor *entropy = args.optional(), *d_log_prob = args.optional(), *d_entropy = args.optional(), *given = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2, "logits are [n, v]");
        const int64_t n = x.size(0), v = x.size(1), ld = pitch(x);
        const int code = code_of(x.scalar_type());
        need(stats.scalar_type() == at::kFloat && stats.is_contiguous() && shape(stats, n, 2), "max_log_sum is float32 [n, 2]");
        if (given) need(given->scalar_type() == x.scalar_type() && shape(*given, n, v), "out is of the logits' type and shape");
        const Tensor out = given ? *given : empty({n, v}, x.scalar_type(), x);
        const int rc = lib.log_probs_bwd(x.data_ptr(), code, n, v, ld, labels_at(labels, n), static_cast<const float *>(stats.data_ptr()), floats_at(entropy, n),
                                         floats_at(d_log_prob, n), floats_at(d_entropy, n), out.data_ptr(), given ? pitch(*given) : v, stream);
        written(given);
        return result(rc, out);
    });
}

// ---- the pointwise layers ---------------------------------------------------------------------------------------------------------
// a program's random state and the operator's site: (state or None, site)
struct Draws {
    const int64_t *state = nullptr;
    uint32_t site = 0;
    explicit Draws(Args &args)
    {
        const Tensor *t = args.optional();
        const int64_t at = args.integer();
        need(at >= 0 && at <= (int64_t)UINT32_MAX, "the site is a 32-bit number");
        site = (uint32_t)at;
        if (!t) return;
        need(t->scalar_type() == at::kLong && t->is_contiguous() && t->numel() == 2, "the random state is int64 [2]: seed, step");
        state = static_cast<const int64_t *>(t->data_ptr());
    }
};
// a batch's offsets or None
struct CloudsOf {
    const int32_t *offsets = nullptr;
    int count = 1;
    explicit CloudsOf(const Tensor *t)
    {
        if (!t) return;
        need(t->scalar_type() == at::kInt && t->dim() == 1 && t->is_contiguous() && t->numel() >= 2 && t->numel() <= INT32_MAX, "offsets are int32 [clouds + 1]");
        offsets = static_cast<const int32_t *>(t->data_ptr());
        count = (int)t->numel() - 1;
    }
};

// (x, residual or None, state, site, p, scope, offsets or None, out or None, device, stream) -> (y,)
PyObject *dropout_fwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const Tensor *residual = args.optional();
        const Draws draws(args);
        const float p = args.number();
        const int scope = args.small();
        const CloudsOf clouds(args.optional());
        const Tensor *given = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2, "x is [n, c]");
        const int64_t n = x.size(0);
        const int c = channels(x), code = code_of(x.scalar_type());
        if (residual) need_rows(*residual, n, c, "the residual is [n, c], contiguous");
        if (given) need_rows(*given, n, c, "out is [n, c], contiguous");
        const at::ScalarType type = residual ? residual->scalar_type() : (given ? given->scalar_type() : x.scalar_type());
        if (given) need(given->scalar_type() == type, "out is of the residual's type");
        const Tensor y = given ? *given : empty({n, c}, type, x);
        const int rc = lib.dropout_fwd(x.data_ptr(), pitch(x), at_of(residual), draws.state, draws.site, p, scope, clouds.offsets, clouds.count, n, c, code,
                                       code_of(type), y.data_ptr(), stream);
        written(given);
        return result(rc, y);
    });
}

// (dy, state, site, p, scope, offsets or None, dtype code (-1: dy's), out or None, device, stream) -> (dx,)
PyObject *dropout_bwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &dy = args.tensor();
        const Draws draws(args);
        const float p = args.number();
        const int scope = args.small();
        const CloudsOf clouds(args.optional());
        const int64_t wanted = args.integer();
        const Tensor *given = args.optional();
        void *stream = args.stream();
        need(dy.dim() == 2 && dy.is_contiguous(), "dy is [n, c], contiguous");
        const int64_t n = dy.size(0);
        const int c = channels(dy);
        if (given) need_rows(*given, n, c, "out is [n, c], contiguous");
        const at::ScalarType type = given ? given->scalar_type() : (wanted < 0 ? dy.scalar_type() : type_of(wanted));
        const Tensor dx = given ? *given : empty({n, c}, type, dy);
        const int rc = lib.dropout_bwd(dy.data_ptr(), draws.state, draws.site, p, scope, clouds.offsets, clouds.count, n, c, code_of(type),
                                       code_of(dy.scalar_type()), dx.data_ptr(), stream);
        written(given);
        return result(rc, dx);
    });
}

// (x, groups, w, b, offsets, act, eps, state, site, p, statistics wanted, out, workspace, device, stream) -> (y, mean_rstd)
PyObject *group_norm_fwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const int groups = args.small();
        const Tensor *w = args.optional(), *b = args.optional();
        const CloudsOf clouds(args.optional());
        const int act = args.small();
        const float eps = args.number();
        const Draws draws(args);
        const float p = args.number();
        const bool keep = args.integer();
        const Tensor *given = args.optional(), *workspace = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2, "x is [n, c]");
        const int64_t n = x.size(0);
        const int c = channels(x), code = code_of(x.scalar_type());
        if (given) {
            need_rows(*given, n, c, "out is [n, c], contiguous");
            need(given->scalar_type() == x.scalar_type(), "out is of x's type");
        }
        const Tensor y = given ? *given : empty({n, c}, x.scalar_type(), x);
        Tensor stats, ws;
        if (keep) stats = empty({clouds.count, groups > 0 ? groups : 1, 2}, at::kFloat, x);
        const size_t bytes = lib.group_norm_workspace_bytes(n, c, clouds.count, groups, 0);
        if (bytes) ws = workspace_of(bytes, workspace, x);
        const int rc = lib.group_norm_fwd(x.data_ptr(), pitch(x), weights(w, c), weights(b, c), clouds.offsets, clouds.count, groups, act, eps, draws.state, draws.site,
                                          p, n, c, code, y.data_ptr(), keep ? static_cast<float *>(stats.data_ptr()) : nullptr, bytes ? ws.data_ptr() : nullptr,
                                          bytes ? ws.nbytes() : 0, stream);
        written(given);
        return result(rc, y, stats);
    });
}

// (dy, x, mean_rstd, w, b, offsets, act, state, site, p, dx wanted, weights' gradients wanted, workspace, device, stream) -> (dx, dw, db)
PyObject *group_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &dy = args.tensor(), &x = args.tensor(), &stats = args.tensor();
        const Tensor *w = args.optional(), *b = args.optional();
        const CloudsOf clouds(args.optional());
        const int act = args.small();
        const Draws draws(args);
        const float p = args.number();
        const bool of_x = args.integer(), of_weights = args.integer();
        const Tensor *workspace = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2, "x is [n, c]");
        const int64_t n = x.size(0);
        const int c = channels(x), code = code_of(x.scalar_type());
        need_rows(dy, n, c, "dy is [n, c], contiguous");
        need(dy.scalar_type() == x.scalar_type(), "dy is of x's type");
        need(stats.scalar_type() == at::kFloat && stats.is_contiguous() && stats.dim() == 3 && stats.size(0) == clouds.count && stats.size(1) >= 1 &&
                 stats.size(1) <= c && stats.size(2) == 2, "mean_rstd is float32 [clouds, groups, 2]");
        const int groups = (int)stats.size(1);
        Tensor dx, dw, db, ws;
        if (of_x) dx = empty({n, c}, x.scalar_type(), x);
        if (of_weights) dw = empty({c}, at::kFloat, x), db = empty({c}, at::kFloat, x);
        const size_t bytes = lib.group_norm_workspace_bytes(n, c, clouds.count, groups, 1);
        if (bytes) ws = workspace_of(bytes, workspace, x);
        auto to = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
        const int rc = lib.group_norm_bwd(dy.data_ptr(), x.data_ptr(), pitch(x), static_cast<const float *>(stats.data_ptr()), weights(w, c), weights(b, c),
                                          clouds.offsets, clouds.count, groups, act, draws.state, draws.site, p, n, c, code, to(dx), static_cast<float *>(to(dw)),
                                          static_cast<float *>(to(db)), to(ws), bytes ? ws.nbytes() : 0, stream);
        return result(rc, dx, dw, db);
    });
}

int64_t mx_row_bytes(int64_t c) { return (c + 31) / 32 * 16; }
int64_t mx_scale_bytes(int64_t c) { return (c + 127) / 128 * 4; }
// Rows of no elements (c = 0) are the columns of a batch without rows.
struct Rows4 {
    const uint8_t *q, *scales;
    int64_t n, c;
    explicit Rows4(Args &args)                                    // (q, scales, c)
    {
        const Tensor &codes = args.tensor(), &exponents = args.tensor();
        c = args.integer();
        need(c >= 0 && c < (1 << 24), "channels outside 0 .. 2^24 - 1");
        n = codes.dim() == 2 ? codes.size(0) : -1;
        need(codes.scalar_type() == at::kByte && exponents.scalar_type() == at::kByte && codes.is_contiguous() && exponents.is_contiguous() &&
                 shape(codes, n, mx_row_bytes(c)) && shape(exponents, n, mx_scale_bytes(c)),
             "q is uint8 [n, pcpp_mx_row_bytes(c)] and scales uint8 [n, pcpp_mx_scale_bytes(c)], both contiguous");
        q = static_cast<const uint8_t *>(codes.data_ptr());
        scales = static_cast<const uint8_t *>(exponents.data_ptr());
    }
};

// (x, rows wanted, columns wanted, state, site, device, stream) -> (q, scales, qt, scales_t)
PyObject *mx_pack(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const bool rows = args.integer(), columns = args.integer();
        const Draws draws(args);
        void *stream = args.stream();
        need(x.dim() == 2, "x is [n, c]");
        need(rows || columns, "neither rows nor columns are wanted");
        const int64_t n = x.size(0), c = x.size(1);
        const int code = code_of(x.scalar_type());
        need(c >= 1 && c < (1 << 24) && (!columns || n < (1 << 24)), "a form's rows have 1 .. 2^24 - 1 elements");
        Tensor q, s, qt, st;
        if (rows) q = empty({n, mx_row_bytes(c)}, at::kByte, x), s = empty({n, mx_scale_bytes(c)}, at::kByte, x);
        if (columns) qt = empty({c, mx_row_bytes(n)}, at::kByte, x), st = empty({c, mx_scale_bytes(n)}, at::kByte, x);
        auto to = [](const Tensor &t) { return t.defined() ? static_cast<uint8_t *>(t.data_ptr()) : nullptr; };
        const int rc = lib.mx_pack(x.data_ptr(), pitch(x), code, n, c, draws.state, draws.site, to(q), to(s), to(qt), to(st), stream);
        return result(rc, q, s, qt, st);
    });
}

// (q, scales, c, dtype code, out or None, device, stream) -> (x,)
PyObject *mx_unpack(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Rows4 rows(args);
        const Tensor &like = THPVariable_Unpack(args.a[0]);
        const int64_t code = args.integer();
        const Tensor *given = args.optional();
        void *stream = args.stream();
        if (given) need_rows(*given, rows.n, rows.c, "out has another shape than the rows, or is not contiguous");
        const Tensor out = given ? *given : empty({rows.n, rows.c}, type_of(code), like);
        const int type = code_of(out.scalar_type());
        const int rc = rows.c == 0 ? PCPP_OK : lib.mx_unpack(rows.q, rows.scales, rows.n, rows.c, out.data_ptr(), type, stream);
        written(given);
        return result(rc, out);
    });
}

const float *bias_at(const Tensor *t, int64_t m)
{
    if (!t) return nullptr;
    need(t->scalar_type() == at::kFloat && t->dim() == 1 && t->size(0) == m && t->is_contiguous(), "the bias is float32 [m]");
    return static_cast<const float *>(t->data_ptr());
}

// (a's q, scales, c, b's q, scales, c, bias, act, dtype code, out, workspace, device, stream) -> (out,)
PyObject *mx_product(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        Rows4 x(args);
        const Tensor &like = THPVariable_Unpack(args.a[0]);
        Rows4 w(args);
        const Tensor *bias = args.optional();
        const int act = args.small();
        const int64_t wanted = args.integer();
        const Tensor *given = args.optional(), *workspace = args.optional();
        void *stream = args.stream();
        need(x.c == w.c, "both sides have the same number of channels");
        if (given) need_rows(*given, x.n, w.n, "out is [n, m], contiguous");
        const Tensor out = given ? *given : empty({x.n, w.n}, type_of(wanted), like);
        Tensor none;
        if (x.c == 0) {                                           // (sums of nothing: those of one block of zeros on either side)
            none = at::zeros({x.n > w.n ? x.n : w.n, mx_row_bytes(1)}, like.options());
            x.q = w.q = x.scales = w.scales = static_cast<const uint8_t *>(none.data_ptr());
            x.c = w.c = 1;
        }
        const size_t bytes = lib.mx_product_workspace_bytes(x.n, w.n, x.c);
        Tensor ws;
        if (bytes) ws = workspace_of(bytes, workspace, like);
        const int rc = lib.mx_product(x.q, x.scales, w.q, w.scales, bias_at(bias, w.n), act, x.n, w.n, x.c, out.data_ptr(), code_of(out.scalar_type()),
                                      bytes ? ws.data_ptr() : nullptr, bytes ? ws.nbytes() : 0, stream);
        written(given);
        return result(rc, out);
    });
}

// (x, w's q, scales, c, bias, act, dtype code (-1: x's), out, workspace, device, stream) -> (out,)
PyObject *mx_linear(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded(a, n_args, [](Args &args) {
        const Tensor &x = args.tensor();
        const Rows4 w(args);
        const Tensor *bias = args.optional();
        const int act = args.small();
        const int64_t wanted = args.integer();
        const Tensor *given = args.optional(), *workspace = args.optional();
        void *stream = args.stream();
        need(x.dim() == 2 && x.size(1) == w.c, "x is [n, k] with the weights' channels");
        const int64_t n = x.size(0);
        if (given) need_rows(*given, n, w.n, "out is [n, m], contiguous");
        const Tensor out = given ? *given : empty({n, w.n}, wanted < 0 ? x.scalar_type() : type_of(wanted), x);
        const size_t bytes = lib.mx_linear_workspace_bytes(n, w.n, w.c);
        Tensor ws;
        if (bytes) ws = workspace_of(bytes, workspace, x);
        const int rc = lib.mx_linear(x.data_ptr(), pitch(x), code_of(x.scalar_type()), w.q, w.scales, bias_at(bias, w.n), act, n, w.n, w.c, out.data_ptr(),
                                     code_of(out.scalar_type()), bytes ? ws.data_ptr() : nullptr, bytes ? ws.nbytes() : 0, stream);
        written(given);
        return result(rc, out);
    });
}

// bind(handle): the library's functions
PyObject *bind(PyObject *, PyObject *arg)
{
    void *handle = PyLong_AsVoidPtr(arg);
    if (!handle && PyErr_Occurred()) return nullptr;
    bool ok = true;
    auto find = [&](auto &f, const char *name) {
        f = reinterpret_cast<std::decay_t<decltype(f)>>(dlsym(handle, name));
        if (!f) ok = false;
    };
    find(lib.act_pack, "pcpp_act_pack");
    find(lib.act_unpack, "pcpp_act_unpack");
    find(lib.mvmr_packed_workspace_bytes, "pcpp_mvmr_packed_workspace_bytes");
    find(lib.mvmr_bwd_weight_packed, "pcpp_mvmr_bwd_weight_packed");
    find(lib.block_norm_fwd, "pcpp_block_norm_fwd");
    find(lib.block_norm_workspace_bytes, "pcpp_block_norm_workspace_bytes");
    find(lib.block_norm_bwd, "pcpp_block_norm_bwd");
    find(lib.log_probs_workspace_bytes, "pcpp_log_probs_workspace_bytes");
    find(lib.log_probs_fwd, "pcpp_log_probs_fwd");
    find(lib.log_probs_bwd, "pcpp_log_probs_bwd");
    find(lib.dropout_fwd, "pcpp_dropout_fwd");
    find(lib.dropout_bwd, "pcpp_dropout_bwd");
    find(lib.group_norm_workspace_bytes, "pcpp_group_norm_workspace_bytes");
    find(lib.group_norm_fwd, "pcpp_group_norm_fwd");
    find(lib.group_norm_bwd, "pcpp_group_norm_bwd");
    find(lib.mx_pack, "pcpp_mx_pack");
    find(lib.mx_unpack, "pcpp_mx_unpack");
    find(lib.mx_product_workspace_bytes, "pcpp_mx_product_workspace_bytes");
    find(lib.mx_product, "pcpp_mx_product");
    find(lib.mx_linear_workspace_bytes, "pcpp_mx_linear_workspace_bytes");
    find(lib.mx_linear, "pcpp_mx_linear");
    if (!ok) {
        PyErr_SetString(PyExc_OSError, "libpcpp.so lacks a function");
        return nullptr;
    }
    Py_RETURN_NONE;
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(act_pack), METHOD(act_unpack), METHOD(weight_packed), METHOD(block_norm_fwd), METHOD(block_norm_bwd), METHOD(log_probs_fwd),
                         METHOD(log_probs_bwd), METHOD(dropout_fwd), METHOD(dropout_bwd), METHOD(group_norm_fwd), METHOD(group_norm_bwd), METHOD(mx_pack), METHOD(mx_unpack),
                         METHOD(mx_product), METHOD(mx_linear), {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls() { return PyModule_Create(&module); }
