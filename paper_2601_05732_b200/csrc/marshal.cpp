// Argument marshalling of the calls around the stack, as a CPython extension: checks the tensors, allocates a call's scratch
// with torch and passes pointers straight to the C ABI.  These calls are made once a token when a model decodes, and through
// ctypes half of such a call's time was spent here (dropout of a small activation 5.9 us, two norms of a token 11.9).
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <new>
#include <string>

#include "../../include/mhclite.h"

namespace {

// The C entry points, taken from the loaded library by name (bind).
struct Entry { const char* name; void* fn; };
enum Id { EMBED_FWD, EMBED_BWD, BLOCK_IN_FWD, BLOCK_IN_BWD, BLOCK_OUT_FWD, BLOCK_OUT_BWD, DROPOUT, CE_FWD, CE_BWD, EMBED_BYTES, BLOCK_BYTES, CE_BYTES,
          DISTILL_FWD, DISTILL_BWD, DISTILL_BYTES, POLICY, PREFERENCE, POLICY_BYTES, PREFERENCE_BYTES, COUNT };
Entry entries[COUNT] = {{"mhclite_embed_fwd", nullptr}, {"mhclite_embed_bwd", nullptr}, {"mhclite_block_in_fwd", nullptr},
                        {"mhclite_block_in_bwd", nullptr}, {"mhclite_block_out_fwd", nullptr}, {"mhclite_block_out_bwd", nullptr},
                        {"mhclite_dropout", nullptr}, {"mhclite_linear_ce_fwd", nullptr}, {"mhclite_linear_ce_bwd", nullptr},
                        {"mhclite_embed_scratch_bytes", nullptr}, {"mhclite_block_scratch_bytes", nullptr},
                        {"mhclite_linear_ce_scratch_bytes", nullptr},
                        {"mhclite_linear_distill_fwd", nullptr}, {"mhclite_linear_distill_bwd", nullptr},
                        {"mhclite_linear_distill_scratch_bytes", nullptr}, {"mhclite_policy_loss", nullptr},
                        {"mhclite_preference_loss", nullptr}, {"mhclite_policy_scratch_bytes", nullptr},
                        {"mhclite_preference_scratch_bytes", nullptr}};
template <typename F> F* entry(Id id, F*) { return reinterpret_cast<F*>(entries[id].fn); }
#define CALL(id, fn, ...) entry(id, &fn)(__VA_ARGS__)

struct Memo { int64_t T = -1, V = -1; size_t bytes = 0; int K = 0; };    // the last sizes whose scratch was asked for
struct Context {
    mhclite_ctx* h;
    int device, n, C;
    Memo embed, block, ce[2], distill[2], policy, preference;
};
const char* kCapsule = "mhclite.context";
Context* context(PyObject* o) { return static_cast<Context*>(PyCapsule_GetPointer(o, kCapsule)); }

std::string text(at::IntArrayRef shape) {
    std::string s = "(";
    for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
    return s + ")";
}

// One call's view of its arguments; `bad` once one has been refused (a Python error is then set).
struct Args {
    Context* c;
    PyObject* const* a;
    bool bad = false;
    explicit Args(PyObject* const* args) : c(nullptr), a(args + 1) {
        if (args[0] == Py_None) PyErr_SetString(PyExc_ValueError, "the context is closed");
        else c = context(args[0]);
        bad = c == nullptr;
    }

    const at::Tensor* tensor(int i, const char* name) {
        if (bad) return nullptr;
        if (!THPVariable_Check(a[i])) {
            PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %s", name, Py_TYPE(a[i])->tp_name);
            bad = true;
            return nullptr;
        }
        return &THPVariable_Unpack(a[i]);
    }
    int64_t rows(int i, const char* name) {                             // length of the first axis
        const at::Tensor* t = tensor(i, name);
        if (!t) return 0;
        if (t->dim() < 1) { PyErr_Format(PyExc_ValueError, "%s: expected at least one axis", name); bad = true; return 0; }
        return t->size(0);
    }
    void* ptr(int i, const char* name, at::ScalarType type, at::IntArrayRef shape) {
        const at::Tensor* t = tensor(i, name);
        if (!t) return nullptr;
        if (t->scalar_type() != type || t->sizes() != shape) {
            const std::string want = text(shape), got = text(t->sizes());
            PyErr_Format(PyExc_ValueError, "%s: expected %s of shape %s, got %s of shape %s", name, c10::toString(type), want.c_str(),
                         c10::toString(t->scalar_type()), got.c_str());
            bad = true;
            return nullptr;
        }
        if (!t->is_cuda() || t->get_device() != c->device || !t->is_contiguous()) {
            PyErr_Format(PyExc_ValueError, "%s: expected a contiguous tensor on cuda:%d", name, c->device);
            bad = true;
            return nullptr;
        }
        return t->data_ptr();
    }
    mhclite_bf16* bf16(int i, const char* name, at::IntArrayRef shape) { return (mhclite_bf16*)ptr(i, name, at::kBFloat16, shape); }
    float* f32(int i, const char* name, at::IntArrayRef shape) { return (float*)ptr(i, name, at::kFloat, shape); }
    int64_t* i64(int i, const char* name, at::IntArrayRef shape) { return (int64_t*)ptr(i, name, at::kLong, shape); }
    bool none(int i) const { return a[i] == Py_None; }
    double real(int i) {
        if (bad) return 0.0;
        const double v = PyFloat_AsDouble(a[i]);
        if (v == -1.0 && PyErr_Occurred()) bad = true;
        return v;
    }
    float number(int i) { return (float)real(i); }
    int truth(int i) {
        if (bad) return 0;
        const int v = PyObject_IsTrue(a[i]);
        if (v < 0) bad = true;
        return v;
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)c->device).stream(); }
    // Scratch on the current stream, which takes it back in stream order (and keeps it to a captured graph), so that calls
    // on several streams and several graphs do not share any.
    at::Tensor scratch(size_t bytes) const {
        if (bytes == 0) return {};
        return at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, (c10::DeviceIndex)c->device));
    }
};
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

PyObject* status(int rc) { return PyLong_FromLong(rc); }

#define TAKE(count)                                                                                                  \
    HANDLE_TH_ERRORS                                                                                                 \
    if (nargs != (count)) { PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", (int)(count) - 1, nargs - 1); return nullptr; } \
    Args x(args);                                                                                                    \
    if (x.bad) return nullptr;                                                                                       \
    const int64_t C = x.c->C;
#define RUN(...)                                                                                                     \
    if (x.bad) return nullptr;                                                                                       \
    void* st = x.stream();                                                                                           \
    int rc;                                                                                                          \
    Py_BEGIN_ALLOW_THREADS                                                                                           \
    rc = __VA_ARGS__;                                                                                                \
    Py_END_ALLOW_THREADS                                                                                             \
    return status(rc);                                                                                               \
    END_HANDLE_TH_ERRORS

PyObject* embed_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {          // ids, E, scale, x0
    TAKE(5)
    const int64_t T = x.rows(0, "ids"), V = x.rows(1, "E");
    if (x.bad) return nullptr;
    const bool f32 = THPVariable_Unpack(x.a[1]).scalar_type() == at::kFloat;
    const int64_t* ids = x.i64(0, "ids", {T});
    const void* E = x.ptr(1, "E", f32 ? at::kFloat : at::kBFloat16, {V, C});
    const float scale = x.number(2);
    mhclite_bf16* x0 = x.bf16(3, "x0", {T, x.c->n, C});
    RUN(CALL(EMBED_FWD, mhclite_embed_fwd, x.c->h, T, V, ids, E, f32, scale, x0, st))
}

PyObject* embed_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {          // ids, g, scale, dE, accumulate
    TAKE(6)
    const int64_t T = x.rows(0, "ids"), V = x.rows(3, "dE");
    const int64_t* ids = x.i64(0, "ids", {T});
    const mhclite_bf16* g = x.bf16(1, "g", {T, x.c->n, C});
    const float scale = x.number(2);
    float* dE = x.f32(3, "dE", {V, C});
    const int acc = x.truth(4);
    if (x.bad) return nullptr;
    Memo& m = x.c->embed;
    if (m.T != T || m.V != V) m = {T, V, CALL(EMBED_BYTES, mhclite_embed_scratch_bytes, (int)C, T, V)};
    const size_t bytes = m.bytes;
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(EMBED_BWD, mhclite_embed_bwd, x.c->h, T, V, ids, g, scale, dE, acc, address(ws), bytes, st))
}

PyObject* block_in_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {       // u, w, eps, v, rstd
    TAKE(6)
    const int64_t T = x.rows(0, "u");
    const mhclite_bf16* u = x.bf16(0, "u", {T, C});
    const float *w = x.f32(1, "w", {C}), eps = x.number(2);
    mhclite_bf16* v = x.bf16(3, "v", {T, C});
    float* rstd = x.f32(4, "rstd", {T});
    RUN(CALL(BLOCK_IN_FWD, mhclite_block_in_fwd, x.c->h, T, u, w, eps, v, rstd, st))
}

size_t block_bytes(Context* c, int64_t T) {
    if (c->block.T != T) c->block = {T, 0, CALL(BLOCK_BYTES, mhclite_block_scratch_bytes, c->C, T)};
    return c->block.bytes;
}

PyObject* block_in_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {       // u, w, rstd, dv, du, dw, accumulate_params
    TAKE(8)
    const int64_t T = x.rows(0, "u");
    const mhclite_bf16* u = x.bf16(0, "u", {T, C});
    const float *w = x.f32(1, "w", {C}), *rstd = x.f32(2, "rstd", {T});
    const mhclite_bf16* dv = x.bf16(3, "dv", {T, C});
    mhclite_bf16* du = x.bf16(4, "du", {T, C});
    float* dw = x.f32(5, "dw", {C});
    const int acc = x.truth(6);
    if (x.bad) return nullptr;
    const size_t bytes = block_bytes(x.c, T);
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(BLOCK_IN_BWD, mhclite_block_in_bwd, x.c->h, T, u, w, rstd, dv, du, dw, acc, address(ws), bytes, st))
}

PyObject* block_out_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {      // o, gate, w, scale, eps, p_drop, rng, y, rstd
    TAKE(10)
    const int64_t T = x.rows(0, "o");
    const mhclite_bf16 *o = x.bf16(0, "o", {T, C}), *gate = x.none(1) ? nullptr : x.bf16(1, "gate", {T, C});
    const float *w = x.f32(2, "w", {C}), *scale = x.none(3) ? nullptr : x.f32(3, "scale", {1}), eps = x.number(4), p = x.number(5);
    const uint64_t* rng = x.none(6) ? nullptr : (const uint64_t*)x.i64(6, "rng", {2});
    mhclite_bf16* y = x.bf16(7, "y", {T, C});
    float* rstd = x.f32(8, "rstd", {T});
    RUN(CALL(BLOCK_OUT_FWD, mhclite_block_out_fwd, x.c->h, T, o, gate, w, scale, eps, p, rng, y, rstd, st))
}

// o, gate, w, scale, rstd, p_drop, rng, dy, d_o, dgate, dw, dscale, accumulate_params
PyObject* block_out_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    TAKE(14)
    const int64_t T = x.rows(0, "o");
    const mhclite_bf16 *o = x.bf16(0, "o", {T, C}), *gate = x.none(1) ? nullptr : x.bf16(1, "gate", {T, C});
    const float *w = x.f32(2, "w", {C}), *scale = x.none(3) ? nullptr : x.f32(3, "scale", {1}), *rstd = x.f32(4, "rstd", {T}), p = x.number(5);
    const uint64_t* rng = x.none(6) ? nullptr : (const uint64_t*)x.i64(6, "rng", {2});
    const mhclite_bf16* dy = x.bf16(7, "dy", {T, C});
    mhclite_bf16 *d_o = x.bf16(8, "d_o", {T, C}), *dgate = x.none(9) ? nullptr : x.bf16(9, "dgate", {T, C});
    float *dw = x.f32(10, "dw", {C}), *dscale = x.none(11) ? nullptr : x.f32(11, "dscale", {1});
    const int acc = x.truth(12);
    if (x.bad) return nullptr;
    const size_t bytes = block_bytes(x.c, T);
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(BLOCK_OUT_BWD, mhclite_block_out_bwd, x.c->h, T, o, gate, w, scale, rstd, p, rng, dy, d_o, dgate, dw, dscale, acc, address(ws),
             bytes, st))
}

PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t nargs) {            // x, p, rng, y
    TAKE(5)
    (void)C;
    const at::Tensor* in = x.tensor(0, "x");
    if (!in) return nullptr;
    const at::IntArrayRef shape = in->sizes();
    const int64_t count = in->numel();
    const mhclite_bf16* from = x.bf16(0, "x", shape);
    const float p = x.number(1);
    const uint64_t* rng = (const uint64_t*)x.i64(2, "rng", {2});
    mhclite_bf16* y = x.bf16(3, "y", shape);
    RUN(CALL(DROPOUT, mhclite_dropout, x.c->h, count, from, p, rng, y, st))
}

size_t ce_bytes(Context* c, int64_t T, int64_t V, int backward) {
    Memo& m = c->ce[backward];
    if (m.T != T || m.V != V) m = {T, V, CALL(CE_BYTES, mhclite_linear_ce_scratch_bytes, c->C, T, V, backward)};
    return m.bytes;
}

PyObject* linear_ce_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {      // h, W, target, logit_scale, loss, lse
    TAKE(7)
    const int64_t T = x.rows(0, "h"), V = x.rows(1, "W");
    const mhclite_bf16 *h = x.bf16(0, "h", {T, C}), *W = x.bf16(1, "W", {V, C});
    const int64_t* target = x.i64(2, "target", {T});
    const float scale = x.number(3);
    float *loss = x.f32(4, "loss", {T}), *lse = x.f32(5, "lse", {T});
    if (x.bad) return nullptr;
    const size_t bytes = ce_bytes(x.c, T, V, 0);
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(CE_FWD, mhclite_linear_ce_fwd, x.c->h, T, V, h, W, target, scale, loss, lse, address(ws), bytes, st))
}

PyObject* linear_ce_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {      // h, W, target, logit_scale, lse, dloss, dh, dW
    TAKE(9)
    const int64_t T = x.rows(0, "h"), V = x.rows(1, "W");
    const mhclite_bf16 *h = x.bf16(0, "h", {T, C}), *W = x.bf16(1, "W", {V, C});
    const int64_t* target = x.i64(2, "target", {T});
    const float scale = x.number(3), *lse = x.f32(4, "lse", {T}), *dloss = x.f32(5, "dloss", {T});
    mhclite_bf16 *dh = x.bf16(6, "dh", {T, C}), *dW = x.bf16(7, "dW", {V, C});
    if (x.bad) return nullptr;
    const size_t bytes = ce_bytes(x.c, T, V, 1);
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(CE_BWD, mhclite_linear_ce_bwd, x.c->h, T, V, h, W, target, scale, lse, dloss, dh, dW, address(ws), bytes, st))
}

// A teacher's entries: ids [T, K] and its logits, fp32 or bf16.
struct Teacher { const int64_t* ids; const void* z; bool f32; int K; };
Teacher teacher(Args& x, int ids, int z, int64_t T) {
    Teacher e = {};
    const at::Tensor *t = x.tensor(ids, "ids"), *v = x.tensor(z, "teacher");
    if (x.bad) return e;
    if (t->dim() != 2 || t->size(1) > 0x7FFFFFFF) {
        PyErr_SetString(PyExc_ValueError, "ids: expected two axes");
        x.bad = true;
        return e;
    }
    e.K = (int)t->size(1);
    e.f32 = v->scalar_type() == at::kFloat;
    e.ids = x.i64(ids, "ids", {T, e.K});
    e.z = x.ptr(z, "teacher", e.f32 ? at::kFloat : at::kBFloat16, {T, e.K});
    return e;
}
size_t distill_bytes(Context* c, int64_t T, int64_t V, int K, int backward) {
    Memo& m = c->distill[backward];
    if (m.T != T || m.V != V || m.K != K) m = {T, V, CALL(DISTILL_BYTES, mhclite_linear_distill_scratch_bytes, c->C, T, V, K, backward), K};
    return m.bytes;
}

// h, W, ids, teacher, logit_scale, temperature, loss, lse, logp
PyObject* linear_distill_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    TAKE(10)
    const int64_t T = x.rows(0, "h"), V = x.rows(1, "W");
    const mhclite_bf16 *h = x.bf16(0, "h", {T, C}), *W = x.bf16(1, "W", {V, C});
    const Teacher e = teacher(x, 2, 3, T);
    const float scale = x.number(4), tau = x.number(5);
    float *loss = x.f32(6, "loss", {T}), *lse = x.f32(7, "lse", {T}), *logp = x.f32(8, "logp", {T, e.K});
    if (x.bad) return nullptr;
    const size_t bytes = distill_bytes(x.c, T, V, e.K, 0);
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(DISTILL_FWD, mhclite_linear_distill_fwd, x.c->h, T, V, e.K, h, W, e.ids, e.z, e.f32, scale, tau, loss, lse, logp, address(ws), bytes, st))
}

// h, W, ids, teacher, logit_scale, temperature, lse, logp, dloss, dh, dW
PyObject* linear_distill_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    TAKE(12)
    const int64_t T = x.rows(0, "h"), V = x.rows(1, "W");
    const mhclite_bf16 *h = x.bf16(0, "h", {T, C}), *W = x.bf16(1, "W", {V, C});
    const Teacher e = teacher(x, 2, 3, T);
    const float scale = x.number(4), tau = x.number(5), *lse = x.f32(6, "lse", {T}), *logp = x.f32(7, "logp", {T, e.K}), *dloss = x.f32(8, "dloss", {T});
    mhclite_bf16 *dh = x.bf16(9, "dh", {T, C}), *dW = x.bf16(10, "dW", {V, C});
    if (x.bad) return nullptr;
    const size_t bytes = distill_bytes(x.c, T, V, e.K, 1);
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(DISTILL_BWD, mhclite_linear_distill_bwd, x.c->h, T, V, e.K, h, W, e.ids, e.z, e.f32, scale, tau, lse, logp, dloss, dh, dW, address(ws), bytes, st))
}

// nll, nll_old, nll_ref, target, starts, adv, token_adv, clip_low, clip_high, kl_weight, mean, loss, stats, dloss, dnll
PyObject* policy_loss(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    TAKE(16)
    (void)C;
    const int64_t T = x.rows(0, "nll"), S = x.rows(11, "loss");
    const float *nll = x.f32(0, "nll", {T}), *old = x.f32(1, "nll_old", {T}), *ref = x.none(2) ? nullptr : x.f32(2, "nll_ref", {T});
    const int64_t *target = x.i64(3, "target", {T}), *starts = x.i64(4, "starts", {S + 1});
    const int each = x.truth(6);
    const float* adv = x.f32(5, "adv", {each ? T : S});
    const double low = x.real(7), high = x.real(8), weight = x.real(9);
    const int mean = x.truth(10);
    float *loss = x.f32(11, "loss", {S}), *stats = x.f32(12, "stats", {S, 3});
    const float* dloss = x.none(13) ? nullptr : x.f32(13, "dloss", {S});
    float* dnll = x.none(14) ? nullptr : x.f32(14, "dnll", {T});
    if (x.bad) return nullptr;
    if (x.none(13) != x.none(14)) { PyErr_SetString(PyExc_ValueError, "dloss and dnll are given both or neither"); return nullptr; }
    Memo& m = x.c->policy;
    if (m.T != T || m.V != S) m = {T, S, CALL(POLICY_BYTES, mhclite_policy_scratch_bytes, T, S)};
    const size_t bytes = m.bytes;
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(POLICY, mhclite_policy_loss, x.c->h, T, S, nll, old, ref, target, starts, adv, each, low, high, weight, mean, dloss, loss, stats, dnll,
             address(ws), bytes, st))
}

// nll, nll_ref, target, starts, beta, margin, smoothing, mean, loss, reward, dloss, dnll
PyObject* preference_loss(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    TAKE(13)
    (void)C;
    const int64_t T = x.rows(0, "nll"), P = x.rows(8, "loss");
    const float *nll = x.f32(0, "nll", {T}), *ref = x.none(1) ? nullptr : x.f32(1, "nll_ref", {T});
    const int64_t *target = x.i64(2, "target", {T}), *starts = x.i64(3, "starts", {2 * P + 1});
    const double beta = x.real(4), margin = x.real(5), smoothing = x.real(6);
    const int mean = x.truth(7);
    float *loss = x.f32(8, "loss", {P}), *reward = x.f32(9, "reward", {P, 2});
    const float* dloss = x.none(10) ? nullptr : x.f32(10, "dloss", {P});
    float* dnll = x.none(11) ? nullptr : x.f32(11, "dnll", {T});
    if (x.bad) return nullptr;
    if (x.none(10) != x.none(11)) { PyErr_SetString(PyExc_ValueError, "dloss and dnll are given both or neither"); return nullptr; }
    Memo& m = x.c->preference;
    if (m.T != T || m.V != P) m = {T, P, CALL(PREFERENCE_BYTES, mhclite_preference_scratch_bytes, T, P)};
    const size_t bytes = m.bytes;
    const at::Tensor ws = x.scratch(bytes);
    RUN(CALL(PREFERENCE, mhclite_preference_loss, x.c->h, T, P, nll, ref, target, starts, beta, margin, smoothing, mean, dloss, loss, reward, dnll,
             address(ws), bytes, st))
}

// bind({name: address}): where the loaded library has the entry points.
PyObject* bind(PyObject*, PyObject* table) {
    for (Entry& e : entries) {
        PyObject* v = PyDict_GetItemString(table, e.name);
        if (!v) { PyErr_SetString(PyExc_KeyError, e.name); return nullptr; }
        e.fn = PyLong_AsVoidPtr(v);
        if (!e.fn) return nullptr;
    }
    Py_RETURN_NONE;
}

// make(handle, device, n, C): what the calls take as their first argument.
PyObject* make(PyObject*, PyObject* args) {
    unsigned long long h;
    int device, n, C;
    if (!PyArg_ParseTuple(args, "Kiii", &h, &device, &n, &C)) return nullptr;
    Context* c = new (std::nothrow) Context{reinterpret_cast<mhclite_ctx*>(h), device, n, C, {}, {}, {}, {}, {}, {}};
    if (!c) return PyErr_NoMemory();
    return PyCapsule_New(c, kCapsule, [](PyObject* o) { delete static_cast<Context*>(PyCapsule_GetPointer(o, kCapsule)); });
}

#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(embed_fwd), METHOD(embed_bwd), METHOD(block_in_fwd), METHOD(block_in_bwd), METHOD(block_out_fwd),
                         METHOD(block_out_bwd), METHOD(dropout), METHOD(linear_ce_fwd), METHOD(linear_ce_bwd), METHOD(linear_distill_fwd), METHOD(linear_distill_bwd),
                         METHOD(policy_loss), METHOD(preference_loss),
                         {"bind", bind, METH_O, nullptr}, {"make", make, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject* torch = PyImport_ImportModule("torch");                   // the tensor class has to be there
    if (!torch) return nullptr;
    PyObject* version = PyObject_GetAttrString(torch, "__version__");
    Py_DECREF(torch);
    const bool same = version && PyUnicode_Check(version) && PyUnicode_CompareWithASCIIString(version, MHCL_TORCH_VERSION) == 0;
    Py_XDECREF(version);
    if (!same) {                                                        // its tensors may be laid out differently
        PyErr_SetString(PyExc_ImportError, "_marshal was built against torch " MHCL_TORCH_VERSION);
        return nullptr;
    }
    return PyModule_Create(&module);
}
