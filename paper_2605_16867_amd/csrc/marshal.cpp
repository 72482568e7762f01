// Argument marshalling of the calls of a serving loop and of a length predictor, in native code: a call of a dozen tensors spends 7 to 9 us
// in the interpreter when each of them is checked there (type, place, layout, size, address), several times what
// the call itself takes to queue its kernels; here it is below one.  What is accepted and what is refused is the same: an
// argument that is not plainly right (a subclass, a wrong type, too short) goes to the binding's own check,
// which raises, or knows it to be right after all.
//
// No kernel and no routing arithmetic here, and no link to the library: the binding hands over the addresses
// of the entry points it has loaded (connect).
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>
#include <vector>

namespace {

using std::int32_t;
using std::int64_t;

struct Entries {
    int (*build_status)(void*, const void*, const void*, const void*, const void*, int64_t, const void*, const void*,
                        const void*, int64_t, void*, void*, void*, void*, void*);
    int (*score_route)(void*, int64_t, const void*, const void*, const void*, const void*, void*, void*, void*, void*, void*);
    int (*score_route_noalloc)(void*, int64_t, const void*, const void*, const void*, const void*, void*, void*, void*, void*);
    int (*score_route_cached)(void*, int64_t, const void*, const void*, const void*, const void*, const void*, const void*,
                              const void*, int64_t, void*, void*, void*, void*, void*);
    int (*route_feedback)(void*, int64_t, int64_t, const void*, const void*, const void*, const void*, void*, void*, void*, void*);
    int (*risk_scan)(void*, const void*, const void*, const void*, const void*, int64_t, const void*, const void*, const void*,
                     int64_t, const void*, void*, void*, void*, void*, void*, void*);
    int (*expert_route)(void*, int64_t, int32_t, const void*, int32_t, const void*, int32_t, int32_t, int32_t, int32_t, float, void*, void*,
                        void*, void*, void*, void*);
    int (*expert_route_backward)(void*, int64_t, int32_t, const void*, int32_t, int32_t, int32_t, float, const void*, const void*, void*, void*);
    int (*expert_plan)(void*, int64_t, int32_t, const void*, void*, void*, void*, void*);
    int (*expert_linear)(void*, int64_t, int32_t, int32_t, int32_t, const void*, const void*, int32_t, const void*, const void*, const void*,
                         int32_t, void*, void*);
    int (*expert_linear_backward)(void*, int64_t, int32_t, int32_t, int32_t, const void*, const void*, int32_t, const void*, const void*,
                                  const void*, const void*, void*, void*, void*, void*, void*);
    int (*expert_combine)(void*, int64_t, int32_t, int32_t, int32_t, const void*, const void*, const void*, void*, void*);
    int (*expert_combine_backward)(void*, int64_t, int32_t, int32_t, int32_t, const void*, const void*, const void*, const void*, void*, void*,
                                   void*);
    int (*clip_gradients)(void*, int32_t, const void* const*, void* const*, const int64_t*, const int32_t*, float, void*, void*);
    int (*token_embed)(void*, int64_t, int32_t, int32_t, int32_t, const void*, const void*, float, void*, void*);
    int (*token_embed_backward)(void*, int64_t, int32_t, int32_t, int32_t, const void*, const void*, float, void*, void*);
    int (*gated_scan)(void*, int64_t, int64_t, int32_t, int32_t, const void*, const void*, int64_t, const void*, int64_t, const void*, void*, void*,
                      void*);
    int (*gated_scan_backward)(void*, int64_t, int64_t, int32_t, int32_t, const void*, const void*, int64_t, const void*, int64_t, const void*,
                               const void*, const void*, const void*, void*, int64_t, void*, int64_t, void*, void*);
    int (*dropout)(void*, int64_t, int32_t, const void*, const void*, double, uint64_t, uint64_t, const void*, void*, void*);
} entries;

PyObject* check_slowly = nullptr;      // (tensor, type code, name, elements or None) -> address or None, or raises

struct Raised {};      // a Python exception is set
struct Unclear {};     // for the binding itself to decide (calls of a length predictor)

constexpr int64_t kAny = -1;

int64_t numel(PyObject* o)
{
    if (THPVariable_CheckExact(o)) return THPVariable_Unpack(o).numel();
    PyObject* n = PyObject_CallMethod(o, "numel", nullptr);
    if (!n) throw Raised{};
    const long long v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

// The address of a contiguous GPU tensor of the type with at least `need` elements; None: null.
void* address(PyObject* o, at::ScalarType type, const char* name, int64_t need = kAny)
{
    if (o == Py_None) return nullptr;
    if (THPVariable_CheckExact(o)) {
        const at::TensorBase& t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.scalar_type() == type && t.is_contiguous() && t.numel() >= need) return t.data_ptr();
    }
    const char* code = type == at::kInt ? "i" : type == at::kFloat ? "f" : type == at::kDouble ? "d" : "B";
    PyObject* r = need == kAny ? PyObject_CallFunction(check_slowly, "OssO", o, code, name, Py_None)
                               : PyObject_CallFunction(check_slowly, "OssL", o, code, name, (long long)need);
    if (!r) throw Raised{};
    void* p = r == Py_None ? nullptr : PyLong_AsVoidPtr(r);
    Py_DECREF(r);
    if (PyErr_Occurred()) throw Raised{};
    return p;
}

void* i32(PyObject* o, const char* name, int64_t need = kAny) { return address(o, at::kInt, name, need); }
void* f32(PyObject* o, const char* name, int64_t need = kAny) { return address(o, at::kFloat, name, need); }
void* f64(PyObject* o, const char* name, int64_t need = kAny) { return address(o, at::kDouble, name, need); }
void* u8(PyObject* o, const char* name, int64_t need = kAny) { return address(o, at::kByte, name, need); }

void* handle(PyObject* o)
{
    if (o == Py_None) return nullptr;
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
}

int64_t integer(PyObject* o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

// torch's current stream on its current device
void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// (the library's calls do not touch Python objects: other threads may run meanwhile)
template <typename... P, typename... A>
PyObject* call(int (*entry)(P...), A... args)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = entry(args...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

template <Py_ssize_t kArgs, PyObject* (*kCall)(PyObject* const*)>
PyObject* guarded(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    if (n != kArgs) { PyErr_Format(PyExc_TypeError, "need %zd arguments, got %zd", kArgs, n); return nullptr; }
    try {
        return kCall(a);
    } catch (const Raised&) {
    } catch (const Unclear&) {
        Py_RETURN_NONE;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// Arguments of each: the handle's address, then what the comment says, in the order of the binding's methods.

// n_inst, act_off, act_prompt, act_gen, act_rem, q_off, q_prompt, q_len, out_act_finish, out_q_finish, out_d, out_rank
PyObject* build_status(PyObject* const* a)
{
    const int64_t M = integer(a[1]), na = numel(a[3]), nq = numel(a[7]);
    void* const act_off = i32(a[2], "act_off", M + 1);
    void* const act_prompt = i32(a[3], "act_prompt");
    void* const act_gen = i32(a[4], "act_gen", na);
    void* const act_rem = i32(a[5], "act_rem", na);
    void* const q_off = i32(a[6], "q_off", M + 1);
    void* const q_prompt = i32(a[7], "q_prompt");
    void* const q_len = i32(a[8], "q_len", nq);
    void* const finish = f32(a[9], "out_act_finish", na);
    void* const q_finish = f32(a[10], "out_q_finish", nq);
    void* const d = f64(a[11], "out_d", M);
    void* const rank = i32(a[12], "out_rank", M);
    return call(entries.build_status, handle(a[0]), act_off, act_prompt, act_gen, act_rem, na, q_off, q_prompt, q_len, nq, finish,
                q_finish, d, rank, stream());
}

struct Requests {
    int64_t n;
    void *ctx0, *len, *budget, *exclude;

    // ctx0, pred_len, budget, exclude_inst
    Requests(PyObject* const* a)
        : n(numel(a[0])), ctx0(i32(a[0], "ctx0")), len(i32(a[1], "pred_len", n)), budget(f32(a[2], "budget", n)),
          exclude(i32(a[3], "exclude_inst", n)) {}
};

struct Choices {
    void *inst, *slack, *fallback;

    // out_inst, out_slack, out_fallback
    Choices(PyObject* const* a, int64_t n)
        : inst(i32(a[0], "out_inst", n)), slack(f32(a[1], "out_slack", n)), fallback(u8(a[2], "out_fallback", n)) {}
};

// n_inst, requests, choices, out_T
PyObject* score_route(PyObject* const* a)
{
    const Requests r(a + 2);
    const Choices c(a + 6, r.n);
    void* const T = f32(a[9], "out_T", r.n * integer(a[1]));
    return call(entries.score_route, handle(a[0]), r.n, r.ctx0, r.len, r.budget, r.exclude, c.inst, c.slack, c.fallback, T, stream());
}

// requests, choices
PyObject* score_route_noalloc(PyObject* const* a)
{
    const Requests r(a + 1);
    const Choices c(a + 5, r.n);
    return call(entries.score_route_noalloc, handle(a[0]), r.n, r.ctx0, r.len, r.budget, r.exclude, c.inst, c.slack, c.fallback, stream());
}

// n_inst, requests, hit_off, hit_inst, hit_len, choices, out_T
PyObject* score_route_cached(PyObject* const* a)
{
    const int64_t nh = numel(a[7]);
    const Requests r(a + 2);
    void* const off = i32(a[6], "hit_off", r.n + 1);
    void* const inst = i32(a[7], "hit_inst");
    void* const len = i32(a[8], "hit_len", nh);
    const Choices c(a + 9, r.n);
    void* const T = f32(a[12], "out_T", r.n * integer(a[1]));
    return call(entries.score_route_cached, handle(a[0]), r.n, r.ctx0, r.len, r.budget, r.exclude, off, inst, len, nh, c.inst, c.slack,
                c.fallback, T, stream());
}

// chunk, requests, choices
PyObject* route_feedback(PyObject* const* a)
{
    const Requests r(a + 2);
    const Choices c(a + 6, r.n);
    return call(entries.route_feedback, handle(a[0]), r.n, integer(a[1]), r.ctx0, r.len, r.budget, r.exclude, c.inst, c.slack, c.fallback,
                stream());
}

// n_inst, act_off, act_prompt, act_gen, act_rem_refreshed, q_off, q_prompt, q_len, act_budget, out_flag, out_finish,
// out_target, out_target_slack, out_n_flagged
PyObject* risk_scan(PyObject* const* a)
{
    const int64_t M = integer(a[1]), na = numel(a[3]), nq = numel(a[7]);
    void* const act_off = i32(a[2], "act_off", M + 1);
    void* const act_prompt = i32(a[3], "act_prompt");
    void* const act_gen = i32(a[4], "act_gen", na);
    void* const act_rem = i32(a[5], "act_rem_refreshed", na);
    void* const q_off = i32(a[6], "q_off", M + 1);
    void* const q_prompt = i32(a[7], "q_prompt");
    void* const q_len = i32(a[8], "q_len", nq);
    void* const budget = f32(a[9], "act_budget", na);
    void* const flag = u8(a[10], "out_flag", na);
    void* const finish = f32(a[11], "out_finish", na);
    void* const target = i32(a[12], "out_target", na);
    void* const slack = f32(a[13], "out_target_slack", na);
    void* const n_flagged = i32(a[14], "out_n_flagged", 1);
    return call(entries.risk_scan, handle(a[0]), act_off, act_prompt, act_gen, act_rem, na, q_off, q_prompt, q_len, nq, budget, flag, finish,
                target, slack, n_flagged, stream());
}

// ---- the calls of a length predictor: None is returned, and nothing called, where an argument is not plainly right,
//      a tensor on another device than the current one and the handle's among them

int64_t here = 0;      // torch's current device, during a call (under the interpreter's lock until the library is called)

template <Py_ssize_t kArgs, PyObject* (*kCall)(PyObject* const*)>
PyObject* on_one_device(PyObject* self, PyObject* const* a, Py_ssize_t n)
{
    here = c10::hip::current_device();
    return guarded<kArgs, kCall>(self, a, n);
}

const at::TensorBase& plain(PyObject* o, int64_t dims = kAny)
{
    if (!THPVariable_CheckExact(o)) throw Unclear{};
    const at::TensorBase& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != here || !t.is_contiguous() || (dims != kAny && t.dim() != dims)) throw Unclear{};
    return t;
}

void* plain(PyObject* o, at::ScalarType type, int64_t need)
{
    if (o == Py_None) return nullptr;
    const at::TensorBase& t = plain(o);
    if (t.scalar_type() != type || t.numel() < need) throw Unclear{};
    return t.data_ptr();
}

int32_t type_code(const at::TensorBase& t)
{
    switch (t.scalar_type()) {
        case at::kFloat: return 0;
        case at::kBFloat16: return 1;
        case at::kHalf: return 2;
        default: throw Unclear{};
    }
}

void must(bool ok)
{
    if (!ok) throw Unclear{};
}

int32_t small(PyObject* o)
{
    const int64_t v = integer(o);
    must(v >= INT32_MIN && v <= INT32_MAX);
    return (int32_t)v;
}

float real(PyObject* o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return (float)v;
}

// A handle's address and device, in a pair; None: null.
void* workspace(PyObject* o)
{
    if (o == Py_None) return nullptr;
    must(PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2 && integer(PyTuple_GET_ITEM(o, 1)) == here);
    return handle(PyTuple_GET_ITEM(o, 0));
}

// n_expert, logits, out_weight, out_expert, out_off, out_slot, out_pos, bias, scoring, n_group, n_group_kept, renormalise, scale
PyObject* expert_route(PyObject* const* a)
{
    const int64_t E = integer(a[1]);
    const at::TensorBase &x = plain(a[2], 2), &e = plain(a[4], 2);
    const int64_t T = x.size(0), k = e.size(1), S = T * k;
    must(x.size(1) == E && e.size(0) == T && k <= INT32_MAX);
    return call(entries.expert_route, workspace(a[0]), T, (int32_t)k, (const void*)x.data_ptr(), type_code(x), (const void*)plain(a[8], at::kFloat, E),
                small(a[9]), small(a[10]), small(a[11]), small(a[12]), real(a[13]), plain(a[3], at::kFloat, S), plain(a[4], at::kInt, S),
                plain(a[5], at::kInt, E + 1), plain(a[6], at::kInt, S), plain(a[7], at::kInt, S), stream());
}

// n_expert, logits, expert, dweight, out_dlogits, scoring, renormalise, scale
PyObject* expert_route_backward(PyObject* const* a)
{
    const at::TensorBase &x = plain(a[2], 2), &e = plain(a[3], 2);
    const int64_t T = x.size(0), k = e.size(1);
    must(x.size(1) == integer(a[1]) && e.size(0) == T && k <= INT32_MAX);
    return call(entries.expert_route_backward, workspace(a[0]), T, (int32_t)k, (const void*)x.data_ptr(), type_code(x), small(a[6]), small(a[7]), real(a[8]),
                (const void*)plain(a[3], at::kInt, T * k), (const void*)plain(a[4], at::kFloat, T * k), plain(a[5], x.scalar_type(), x.numel()), stream());
}

// n_expert, expert, out_off, out_slot, out_pos
PyObject* expert_plan(PyObject* const* a)
{
    const at::TensorBase& e = plain(a[2], 2);
    must(e.size(1) <= INT32_MAX);
    return call(entries.expert_plan, workspace(a[0]), (int64_t)e.size(0), (int32_t)e.size(1), (const void*)plain(a[2], at::kInt, 0),
                plain(a[3], at::kInt, integer(a[1]) + 1), plain(a[4], at::kInt, e.numel()), plain(a[5], at::kInt, e.numel()), stream());
}

struct Layer {
    int64_t E, n;
    int32_t I, O, type, top_k;
    at::ScalarType scalar;
    const void *off, *slot, *x, *w;

    // n_expert, x, w; what has a row per position; off, slot, top_k
    Layer(PyObject* n_expert, PyObject* x_, PyObject* w_, PyObject* by_position, PyObject* off_, PyObject* slot_, PyObject* top_k_)
    {
        const at::TensorBase &x_t = plain(x_, 2), &w_t = plain(w_), &p = plain(by_position, 2);
        const int64_t N = integer(n_expert), d = w_t.dim();
        E = off_ == Py_None ? 1 : N;
        must(d == 3 ? w_t.size(0) == E : d == 2 && off_ == Py_None);
        must(w_t.size(d - 1) <= INT32_MAX && w_t.size(d - 2) <= INT32_MAX);
        I = (int32_t)w_t.size(d - 1);
        O = (int32_t)w_t.size(d - 2);
        n = p.size(0);
        top_k = small(top_k_);
        type = type_code(x_t);
        scalar = x_t.scalar_type();
        must(p.size(1) == O && x_t.size(1) == I && w_t.scalar_type() == scalar && p.scalar_type() == scalar);
        must(slot_ == Py_None ? x_t.size(0) == n : top_k >= 1 && x_t.size(0) == (n + top_k - 1) / top_k);
        off = plain(off_, at::kInt, N + 1);
        slot = plain(slot_, at::kInt, n);
        x = x_t.data_ptr();
        w = w_t.data_ptr();
    }
};

// n_expert, x, w, out_y, bias, off, slot, top_k, relu
PyObject* expert_linear(PyObject* const* a)
{
    const Layer l(a[1], a[2], a[3], a[4], a[6], a[7], a[8]);
    return call(entries.expert_linear, workspace(a[0]), l.n, l.I, l.O, l.type, l.off, l.slot, l.top_k, l.x, l.w, (const void*)plain(a[5], l.scalar, l.E * l.O),
                small(a[9]), plain(a[4], l.scalar, l.n * l.O), stream());
}

// n_expert, x, w, dy, out_dx, out_dw, out_db, y, out_dz, off, slot, top_k
PyObject* expert_linear_backward(PyObject* const* a)
{
    const Layer l(a[1], a[2], a[3], a[4], a[10], a[11], a[12]);
    const int64_t of_y = l.n * l.O;
    return call(entries.expert_linear_backward, workspace(a[0]), l.n, l.I, l.O, l.type, l.off, l.slot, l.top_k, l.x, l.w, (const void*)plain(a[8], l.scalar, of_y),
                (const void*)plain(a[4], l.scalar, of_y), plain(a[9], l.scalar, of_y), plain(a[5], l.scalar, l.n * l.I),
                plain(a[6], l.scalar, l.E * l.O * l.I), plain(a[7], l.scalar, l.E * l.O), stream());
}

// y, pos, out, weight
PyObject* expert_combine(PyObject* const* a)
{
    const at::TensorBase &pos = plain(a[2], 2), &out = plain(a[3], 2);
    const int64_t T = pos.size(0), S = pos.numel(), O = out.size(1);
    must(out.size(0) == T && O <= INT32_MAX && pos.size(1) <= INT32_MAX);
    return call(entries.expert_combine, workspace(a[0]), T, (int32_t)pos.size(1), (int32_t)O, type_code(out), (const void*)plain(a[4], at::kFloat, S),
                (const void*)plain(a[2], at::kInt, S), (const void*)plain(a[1], out.scalar_type(), S * O), out.data_ptr(), stream());
}

// dout, y, slot, out_dy, weight, out_dweight
PyObject* expert_combine_backward(PyObject* const* a)
{
    const at::TensorBase &d = plain(a[1], 2), &slot = plain(a[3]);
    const int64_t T = d.size(0), O = d.size(1), S = slot.numel();
    must(T > 0 && S % T == 0 && S / T <= INT32_MAX && O <= INT32_MAX);
    return call(entries.expert_combine_backward, workspace(a[0]), T, (int32_t)(S / T), (int32_t)O, type_code(d), (const void*)plain(a[5], at::kFloat, S),
                (const void*)plain(a[3], at::kInt, S), (const void*)plain(a[2], d.scalar_type(), S * O), (const void*)d.data_ptr(),
                plain(a[4], d.scalar_type(), S * O), plain(a[6], at::kFloat, S), stream());
}

// grads, max_norm, out_norm, out (lists of as many)
PyObject* clip_gradients(PyObject* const* a)
{
    must(PyList_CheckExact(a[1]) && PyList_CheckExact(a[4]));
    const Py_ssize_t n = PyList_GET_SIZE(a[1]);
    must(PyList_GET_SIZE(a[4]) == n && n <= INT32_MAX);
    std::vector<const void*> grad(n);
    std::vector<void*> out(n);
    std::vector<int64_t> count(n);
    std::vector<int32_t> type(n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::TensorBase& g = plain(PyList_GET_ITEM(a[1], i));
        grad[i] = g.data_ptr();
        count[i] = g.numel();
        type[i] = type_code(g);
        must(PyList_GET_ITEM(a[4], i) != Py_None);
        out[i] = plain(PyList_GET_ITEM(a[4], i), g.scalar_type(), count[i]);
    }
    return call(entries.clip_gradients, workspace(a[0]), (int32_t)n, (const void* const*)grad.data(), (void* const*)out.data(), (const int64_t*)count.data(),
                (const int32_t*)type.data(), real(a[2]), plain(a[3], at::kFloat, 1), stream());
}

// A whole number of 64 bits without a sign.
uint64_t bits(PyObject* o)
{
    must(PyLong_CheckExact(o));
    const unsigned long long v = PyLong_AsUnsignedLongLong(o);
    if (v == (unsigned long long)-1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Unclear{};
    }
    return v;
}

int32_t size32(int64_t n)
{
    must(n <= INT32_MAX);
    return (int32_t)n;
}

// A dense tensor of these sizes; None: null.
void* sized(PyObject* o, at::ScalarType type, int64_t n, int64_t width)
{
    if (o == Py_None) return nullptr;
    const at::TensorBase& t = plain(o, 2);
    must(t.scalar_type() == type && t.size(0) == n && t.size(1) == width);
    return t.data_ptr();
}

// token, rows of tokens, rows of the table, scale
template <typename Entry>
PyObject* embed(Entry entry, PyObject* handle_, PyObject* token_, PyObject* in_, PyObject* rows_, PyObject* table_, PyObject* out_, PyObject* scale)
{
    const at::TensorBase &token = plain(token_, 1), &table = plain(table_, 2);
    const int64_t n = token.numel(), V = table.size(0), W = table.size(1);
    must(token.scalar_type() == at::kInt);
    (void)sized(rows_, table.scalar_type(), n, W);
    const at::TensorBase &in = plain(in_, 2), &out = plain(out_, 2);
    return call(entry, workspace(handle_), n, size32(V), size32(W), type_code(table), (const void*)token.data_ptr(), (const void*)in.data_ptr(),
                real(scale), (void*)out.data_ptr(), stream());
}

// token, table, out, scale
PyObject* token_embed(PyObject* const* a) { return embed(entries.token_embed, a[0], a[1], a[2], a[3], a[2], a[3], a[4]); }

// token, dout, out_dtable, scale
PyObject* token_embed_backward(PyObject* const* a) { return embed(entries.token_embed_backward, a[0], a[1], a[2], a[2], a[3], a[3], a[4]); }

// Rows of one type that need not be next to each other.
struct Rows {
    void* at;
    int64_t stride;

    Rows(PyObject* o, at::ScalarType type, int64_t n, int64_t width)
    {
        must(THPVariable_CheckExact(o));
        const at::TensorBase& t = THPVariable_Unpack(o);
        must(t.is_cuda() && t.get_device() == here && t.dim() == 2 && t.scalar_type() == type && t.size(0) == n && t.size(1) == width);
        must(n > 0 && width > 0 && (width == 1 || t.stride(1) == 1));
        stride = n > 1 ? t.stride(0) : width;
        must(stride >= width);
        at = t.data_ptr();
    }
};

struct Sequences {
    int64_t n, W, S;
    at::ScalarType scalar;
    int32_t type;
    const void* off;

    // gate, off
    Sequences(PyObject* gate_, PyObject* off_)
    {
        must(THPVariable_CheckExact(gate_));
        const at::TensorBase& gate = THPVariable_Unpack(gate_);
        must(gate.dim() == 2);
        n = gate.size(0);
        W = gate.size(1);
        scalar = gate.scalar_type();
        type = type_code(gate);
        off = nullptr;
        S = n;
        if (off_ != Py_None) {
            const at::TensorBase& t = plain(off_, 1);
            must(t.scalar_type() == at::kInt && t.numel() > 0);
            off = t.data_ptr();
            S = t.numel() - 1;
        }
    }
};

// gate, x, out_y, off, h0, out_h
PyObject* gated_scan(PyObject* const* a)
{
    const Sequences q(a[1], a[4]);
    const Rows gate(a[1], q.scalar, q.n, q.W), x(a[2], q.scalar, q.n, q.W);
    return call(entries.gated_scan, workspace(a[0]), q.n, q.S, size32(q.W), q.type, q.off, (const void*)gate.at, gate.stride, (const void*)x.at, x.stride,
                (const void*)sized(a[5], at::kFloat, q.S, q.W), sized(a[3], q.scalar, q.n, q.W), sized(a[6], at::kFloat, q.S, q.W), stream());
}

// gate, x, y, out_dgate, out_dx, off, h0, dy, dh, out_dh0
PyObject* gated_scan_backward(PyObject* const* a)
{
    const Sequences q(a[1], a[6]);
    const Rows gate(a[1], q.scalar, q.n, q.W), x(a[2], q.scalar, q.n, q.W), dgate(a[4], q.scalar, q.n, q.W), dx(a[5], q.scalar, q.n, q.W);
    return call(entries.gated_scan_backward, workspace(a[0]), q.n, q.S, size32(q.W), q.type, q.off, (const void*)gate.at, gate.stride, (const void*)x.at,
                x.stride, (const void*)sized(a[3], q.scalar, q.n, q.W), (const void*)sized(a[7], at::kFloat, q.S, q.W),
                (const void*)sized(a[8], q.scalar, q.n, q.W), (const void*)sized(a[9], at::kFloat, q.S, q.W), dgate.at, dgate.stride, dx.at, dx.stride,
                sized(a[10], at::kFloat, q.S, q.W), stream());
}

// x, out, rate, seed, offset, residual, offset_add
PyObject* dropout(PyObject* const* a)
{
    const at::TensorBase &x = plain(a[1]), &out = plain(a[2]);
    must(out.sizes() == x.sizes() && out.scalar_type() == x.scalar_type());
    const void* residual = nullptr;
    if (a[6] != Py_None) {
        const at::TensorBase& r = plain(a[6]);
        must(r.sizes() == x.sizes() && r.scalar_type() == x.scalar_type());
        residual = r.data_ptr();
    }
    const double rate = PyFloat_AsDouble(a[3]);
    if (rate == -1 && PyErr_Occurred()) throw Raised{};
    return call(entries.dropout, workspace(a[0]), (int64_t)x.numel(), type_code(x), (const void*)x.data_ptr(), residual, rate, bits(a[4]), bits(a[5]),
                (const void*)plain(a[7], at::kLong, 1), (void*)out.data_ptr(), stream());
}

// check_slowly, then the addresses of the entry points in the order of Entries
PyObject* connect(PyObject* const* a)
{
    void** const to = reinterpret_cast<void**>(&entries);
    for (size_t i = 0; i < sizeof entries / sizeof(void*); ++i) to[i] = handle(a[1 + i]);
    Py_INCREF(a[0]);
    Py_XSETREF(check_slowly, a[0]);
    Py_RETURN_NONE;
}

#define GR_METHOD(name, n) {#name, (PyCFunction)(void (*)(void))guarded<n, name>, METH_FASTCALL, nullptr}
#define GR_METHOD_HERE(name, n) {#name, (PyCFunction)(void (*)(void))on_one_device<n, name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {GR_METHOD(build_status, 13), GR_METHOD(score_route, 10), GR_METHOD(score_route_noalloc, 8),
                         GR_METHOD(score_route_cached, 13), GR_METHOD(route_feedback, 9), GR_METHOD(risk_scan, 15),
                         GR_METHOD_HERE(expert_route, 14), GR_METHOD_HERE(expert_route_backward, 9), GR_METHOD_HERE(expert_plan, 6),
                         GR_METHOD_HERE(expert_linear, 10), GR_METHOD_HERE(expert_linear_backward, 13), GR_METHOD_HERE(expert_combine, 5),
                         GR_METHOD_HERE(expert_combine_backward, 7), GR_METHOD_HERE(clip_gradients, 5),
                         GR_METHOD_HERE(token_embed, 5), GR_METHOD_HERE(token_embed_backward, 5), GR_METHOD_HERE(gated_scan, 7),
                         GR_METHOD_HERE(gated_scan_backward, 11), GR_METHOD_HERE(dropout, 8),
                         GR_METHOD(connect, 20), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_goodroute_marshal(void) { return PyModule_Create(&module); }
