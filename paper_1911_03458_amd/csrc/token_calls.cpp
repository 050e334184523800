// The Python calls of the operators along a sequence of tokens, natively: checks, allocations (outputs, scratch memory) and
// the launch in one call (see torch_calls.cpp, whose module this is part of).  Which operands a call has -- types, shapes,
// strided dimensions, inputs and outputs -- comes from tokens.py once per plan; a call that is not of the ordinary form is
// not judged here: token_call() returns None and the general path takes it.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <new>

#include "merit_tokens.h"

namespace {

constexpr int MOST = 24;

typedef merit_status (*Entry)(const merit_token_plan *, const merit_view *, void *, int64_t, void *);
template <typename A, merit_status (*F)(const merit_token_plan *, const A *, void *, int64_t, void *)>
merit_status entry(const merit_token_plan *plan, const merit_view *v, void *ws, int64_t bytes, void *stream)
{
    return F(plan, reinterpret_cast<const A *>(v), ws, bytes, stream);      // (an argument struct is its views, in order)
}
constexpr struct {
    const char *name;
    Entry run;
    size_t views;
} kOps[] = {
#define OP(f) {#f, entry<f##_args, f>, sizeof(f##_args) / sizeof(merit_view)}
    OP(merit_group_norm), OP(merit_group_norm_backward), OP(merit_causal_conv), OP(merit_causal_conv_backward),
    OP(merit_causal_conv_step), OP(merit_scan), OP(merit_scan_backward), OP(merit_scan_step)
#undef OP
};
constexpr int OPS = sizeof(kOps) / sizeof(kOps[0]);

enum Kind { TYPE, PARAM, F32, I32 };
enum Role { IN, OPT, OUT, OUT_OPT };
struct Operand {
    Kind kind;
    Role role;
    int n, lead;
    int64_t shape[4];
    at::IntArrayRef ref() const { return at::IntArrayRef(shape, static_cast<size_t>(n)); }
};
struct Spec {
    int op;
    merit_token_plan *plan;
    int dtype;
    at::ScalarType type;
    int64_t scratch;
    int n;
    Operand operand[MOST];
};

const char *kSpec = "merit.token_spec";

void free_spec(PyObject *capsule) { delete static_cast<Spec *>(PyCapsule_GetPointer(capsule, kSpec)); }

bool read_spec(PyObject *const *args, Spec *s)
{
    s->op = static_cast<int>(PyLong_AsLong(args[0]));
    s->plan = static_cast<merit_token_plan *>(PyLong_AsVoidPtr(args[1]));
    s->dtype = static_cast<int>(PyLong_AsLong(args[2]));
    s->scratch = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred() || s->op < 0 || s->op >= OPS || !PyTuple_Check(args[4])) return false;
    s->type = s->dtype == MERIT_F32 ? at::kFloat : s->dtype == MERIT_F16 ? at::kHalf : at::kBFloat16;
    s->n = static_cast<int>(PyTuple_GET_SIZE(args[4]));
    if (s->n > MOST || static_cast<size_t>(s->n) != kOps[s->op].views) return false;
    for (int i = 0; i < s->n; ++i) {
        int kind, lead, role;
        PyObject *shape;
        if (!PyArg_ParseTuple(PyTuple_GET_ITEM(args[4], i), "iO!ii", &kind, &PyTuple_Type, &shape, &lead, &role)) return false;
        Operand &o = s->operand[i];
        o.kind = static_cast<Kind>(kind);
        o.role = static_cast<Role>(role);
        o.lead = lead;
        if (PyTuple_GET_SIZE(shape) > 4 || lead > 2) return false;
        o.n = static_cast<int>(PyTuple_GET_SIZE(shape));
        for (int k = 0; k < o.n; ++k) o.shape[k] = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, k));
        if (PyErr_Occurred()) return false;
    }
    return true;
}

// token_spec(op, handle, dtype, scratch bytes, ((kind, shape, leading strides, role), ...)) -> capsule
PyObject *make_spec(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    Spec *s = n == 5 ? new (std::nothrow) Spec() : nullptr;
    if (s) {
        if (read_spec(args, s)) {
            PyObject *c = PyCapsule_New(s, kSpec, free_spec);
            if (c) return c;
        }
        delete s;
    }
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "token_spec(op, handle, dtype, scratch bytes, operands)");
    return nullptr;
}

constexpr c10::DispatchKeySet kNotPlain({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched,
                                         c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
                                         c10::DispatchKey::Conjugate, c10::DispatchKey::Negative});

// The device tensor in `o` as operand `q`, or nullptr
const at::Tensor *plain(PyObject *o, const Spec &s, const Operand &q, merit_view *v)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda()) return nullptr;
    const c10::TensorImpl *impl = t.unsafeGetTensorImpl();
    if (impl->key_set().has_any(kNotPlain) || !impl->has_storage() || impl->has_symbolic_sizes_strides()) return nullptr;
    const at::ScalarType type = t.scalar_type();
    const bool fits = q.kind == TYPE ? type == s.type : q.kind == PARAM ? type == s.type || type == at::kFloat
                      : q.kind == F32 ? type == at::kFloat : type == at::kInt;
    if (!fits || t.sizes() != q.ref()) return nullptr;
    int64_t dense = 1;
    const at::IntArrayRef st = t.strides();
    for (int i = q.n - 1; i >= q.lead; --i) {
        if (q.shape[i] > 1 && st[i] != dense && t.numel()) return nullptr;
        dense *= q.shape[i];
    }
    v->data = t.data_ptr();
    v->stride[0] = q.lead > 0 ? st[0] : 0;
    v->stride[1] = q.lead > 1 ? st[1] : 0;
    v->dtype = type == at::kFloat ? MERIT_F32 : q.kind == I32 ? 0 : s.dtype;
    v->reserved = 0;
    return &t;
}

// token_call(spec, wanted outputs, operand...) -> tuple of the outputs; the status as an int if the library refuses;
// None if the call is not of the ordinary form
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n < 2) {
        PyErr_SetString(PyExc_TypeError, "token_call(spec, wanted outputs, operand...)");
        return nullptr;
    }
    const Spec *s = static_cast<const Spec *>(PyCapsule_GetPointer(args[0], kSpec));
    if (!s) return nullptr;
    const long long want = PyLong_AsLongLong(args[1]);
    if (want == -1 && PyErr_Occurred()) return nullptr;
    if (n != 2 + s->n) {
        PyErr_SetString(PyExc_TypeError, "token_call: another number of operands");
        return nullptr;
    }
    if (c10::impl::TorchDispatchModeTLS::any_modes_set() || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;

    merit_view v[MOST] = {};
    const at::Tensor *first = nullptr;
    for (int i = 0; i < s->n; ++i) {
        if (args[2 + i] == Py_None) {
            if (s->operand[i].role == IN) Py_RETURN_NONE;
            continue;
        }
        const at::Tensor *t = plain(args[2 + i], *s, s->operand[i], v + i);
        if (!t || (first && t->device() != first->device())) Py_RETURN_NONE;
        if (!first) first = t;
    }
    if (!first || first->device().index() != c10::hip::current_device()) Py_RETURN_NONE;

    const at::TensorOptions opts = at::TensorOptions().device(first->device());
    at::Tensor made[MOST], scratch;
    for (int i = 0; i < s->n; ++i) {
        const Operand &q = s->operand[i];
        if (q.role < OUT || args[2 + i] != Py_None || !(want >> i & 1)) continue;
        made[i] = at::empty(q.ref(), opts.dtype(q.kind == F32 ? at::kFloat : s->type));
        v[i].data = made[i].data_ptr();
        v[i].stride[0] = q.lead > 0 ? made[i].stride(0) : 0;
        v[i].stride[1] = q.lead > 1 ? made[i].stride(1) : 0;
        v[i].dtype = q.kind == F32 ? MERIT_F32 : s->dtype;
    }
    if (s->scratch) scratch = at::empty({s->scratch}, opts.dtype(at::kByte));
    void *ws = s->scratch ? scratch.data_ptr() : nullptr;
    void *stream = c10::hip::getCurrentHIPStream().stream();

    merit_status st = MERIT_ERR_INVALID_ARG;
    Py_BEGIN_ALLOW_THREADS
    st = kOps[s->op].run(s->plan, v, ws, s->scratch, stream);
    Py_END_ALLOW_THREADS
    if (st != MERIT_OK) return PyLong_FromLong(st);

    int outs = 0;
    for (int i = 0; i < s->n; ++i) outs += s->operand[i].role >= OUT;
    PyObject *r = PyTuple_New(outs);
    for (int i = 0, k = 0; r && i < s->n; ++i) {
        if (s->operand[i].role < OUT) continue;
        PyObject *o = args[2 + i];
        if (o == Py_None && made[i].defined()) {
            o = THPVariable_Wrap(std::move(made[i]));
            if (!o) {
                Py_CLEAR(r);
                break;
            }
        } else {
            Py_INCREF(o);
        }
        PyTuple_SET_ITEM(r, k++, o);
    }
    return r;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"token_spec", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(make_spec)), METH_FASTCALL, nullptr},
    {"token_call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

}  // namespace

// Adds these calls to the module: TOKEN_OPS and two functions
bool merit_add_token_calls(PyObject *module)
{
    if (PyModule_AddFunctions(module, methods) != 0) return false;
    PyObject *ops = PyDict_New();
    bool ok = ops != nullptr;
    for (int i = 0; i < OPS && ok; ++i) {
        PyObject *k = PyLong_FromLong(i);
        ok = k && PyDict_SetItemString(ops, kOps[i].name, k) == 0;
        Py_XDECREF(k);
    }
    ok = ok && PyObject_SetAttrString(module, "TOKEN_OPS", ops) == 0;
    Py_XDECREF(ops);
    return ok;
}
