// Python entry points of the calls on pages.  A step of a served batch calls each of them once per decoder layer, for kernels of a
// few microseconds: through ctypes and Python's own checks a call cost 23 to 37 us of the host's time, more than the kernels of a
// small batch take, so these calls are checked, allocated for and launched here (4 to 9 us, one or two launches among them).
//
// Everything is as in the C entry points (include/locret.h), on torch's current stream; what can be seen of the tensors is checked
// and refused with ValueError, what the library returns is raised as LocretError.  Autograd records none of the calls; tensors that
// they write in place count as changed.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <structmember.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/locret.h"

namespace {

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };   // ValueError
struct Raised {};                                                                   // a Python exception is set

[[noreturn]] void refuse(const std::string &why) { throw Refused(why); }

PyObject *module_self = nullptr;

void check(int code, const char *what) {
  if (code == LOCRET_OK) return;
  PyObject *type = PyObject_GetAttrString(module_self, "LocretError");
  if (type) {
    PyObject *e = PyObject_CallFunction(type, "is", code, what);
    if (e) { PyErr_SetObject(type, e); Py_DECREF(e); }
    Py_DECREF(type);
  }
  throw Raised();
}

// A function's argument names, as the interned strings that its callers' keywords are (compared by address first: by letters
// alone, ten keywords took longer than the checks).
template <int N>
struct Names {
  PyObject *interned[N];
  explicit Names(const char *const (&names)[N]) {
    for (int i = 0; i < N; i++) {
      interned[i] = PyUnicode_InternFromString(names[i]);   // (kept for the life of the process)
      if (!interned[i]) throw Raised();
    }
  }
  int find(PyObject *name) const {
    for (int i = 0; i < N; i++)
      if (interned[i] == name) return i;
    for (int i = 0; i < N; i++)
      if (PyUnicode_Compare(interned[i], name) == 0) return i;
    return -1;
  }
};

// Positional and keyword arguments, by name; the first `required` have to be there.  None counts as absent.
template <int N>
struct Args {
  PyObject *v[N] = {};
  Args(const char *func, const Names<N> &names, int required, PyObject *const *args, Py_ssize_t n, PyObject *kwnames) {
    if (n > N) fail(func, "takes at most " + std::to_string(N) + " arguments");
    for (Py_ssize_t i = 0; i < n; i++) v[i] = args[i];
    const Py_ssize_t n_kw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    for (Py_ssize_t k = 0; k < n_kw; k++) {
      PyObject *name = PyTuple_GET_ITEM(kwnames, k);
      const int at = names.find(name);
      if (at < 0 || v[at]) fail(func, std::string(at < 0 ? "got an unexpected argument '" : "got two values for '") + PyUnicode_AsUTF8(name) + "'");
      v[at] = args[n + k];
    }
    for (int i = 0; i < N; i++) {
      if (v[i] == Py_None) v[i] = nullptr;
      if (!v[i] && i < required) fail(func, std::string("needs '") + PyUnicode_AsUTF8(names.interned[i]) + "'");
    }
  }
  [[noreturn]] static void fail(const char *func, const std::string &why) {
    PyErr_SetString(PyExc_TypeError, (std::string(func) + "() " + why).c_str());
    throw Raised();
  }
};

const at::Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
    throw Raised();
  }
  return THPVariable_Unpack(o);
}
long long integer(PyObject *o, long long dflt) {
  if (!o) return dflt;
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) throw Raised();
  return x;
}
int integer32(PyObject *o, int dflt, const char *what) {
  const long long x = integer(o, dflt);
  if (x < INT32_MIN || x > INT32_MAX) refuse(std::string(what) + " does not fit 32 bits");
  return (int)x;
}
double number(PyObject *o, double dflt) {
  if (!o) return dflt;
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) throw Raised();
  return x;
}
bool truth(PyObject *o) {
  if (!o) return false;
  const int x = PyObject_IsTrue(o);
  if (x < 0) throw Raised();
  return x != 0;
}

// The device of a call's tensors: the current one.
struct Where {
  c10::Device device;
  void *stream;
  explicit Where(const at::Tensor &t, const char *what) : device(t.device()), stream(nullptr) {
    if (!t.is_cuda() || t.get_device() != c10::cuda::current_device())
      refuse(std::string(what) + " must be a tensor of the current CUDA device");
    stream = c10::cuda::getCurrentCUDAStream(t.get_device()).stream();
  }
};
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Where &w) {
  return at::detail::empty_cuda(shape, type, w.device, c10::nullopt);   // (at::empty without the dispatcher)
}

// words (lengths, tables, positions ...): a type, a number of dimensions, the last one contiguous
void *words(PyObject *o, const char *what, at::ScalarType type, int dim, const Where &w, const at::Tensor **out = nullptr) {
  const at::Tensor &t = tensor(o, what);
  if (t.scalar_type() != type || t.dim() != dim || t.device() != w.device || (dim && t.size(dim - 1) > 1 && t.stride(dim - 1) != 1))
    refuse(std::string(what) + " must be a tensor of type " + c10::toString(type) + " with " + std::to_string(dim) +
           " dimension(s) on " + w.device.str() + ", contiguous in the last one");
  if (out) *out = &t;
  return t.data_ptr();
}
int32_t *status_word(PyObject *o, const Where &w) {
  if (!o) return nullptr;
  const at::Tensor &t = tensor(o, "status");
  if (t.scalar_type() != at::kInt || t.numel() < 1 || t.device() != w.device)
    refuse("status must be an int32 tensor on " + w.device.str());
  return static_cast<int32_t *>(t.data_ptr());
}
// The calls record nothing for autograd: an input that requires gradients would give outputs that silently have none.
void no_graph(const at::Tensor &t, const char *what) {
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse(std::string(what) + " requires gradients, which this call does not record: call it under torch.no_grad() or in the forward "
                               "of a torch.autograd.Function (gradients of norm_rope: norm_rope_grad)");
}
// What a call has written in place, for autograd's check that nothing saved for a backward pass has changed since.
void changed(const at::Tensor &t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void changed(PyObject *o) {
  if (o) changed(THPVariable_Unpack(o));
}
// [tokens or requests, heads, d] of any strides whose last dimension is contiguous
const at::Tensor &heads(PyObject *o, const char *what, at::ScalarType type, const Where &w) {
  const at::Tensor &t = tensor(o, what);
  if (t.dim() != 3 || t.scalar_type() != type || t.device() != w.device || (t.size(2) > 1 && t.stride(2) != 1))
    refuse(std::string(what) + " must have three dimensions (tokens, heads, d), type " + c10::toString(type) + ", lie on " +
           w.device.str() + " and be contiguous in the last dimension");
  return t;
}
// where a call writes: no two elements in one place
const at::Tensor &written(PyObject *o, const char *what, at::ScalarType type, const Where &w) {
  const at::Tensor &t = heads(o, what, type, w);
  for (int i = 0; i < 2; i++)
    if (t.size(i) > 1 && t.stride(i) == 0) refuse(std::string(what) + " is an expanded tensor");
  no_graph(t, what);
  return t;
}
void same_shape(const at::Tensor &a, const at::Tensor &b, const char *what) {
  if (a.sizes() != b.sizes()) refuse(std::string(what) + " do not have the same shape");
}
int dtype_code(at::ScalarType t) { return t == at::kBFloat16 ? LOCRET_BF16 : t == at::kHalf ? LOCRET_FP16 : -1; }

PyObject *wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }

template <typename F>
PyObject *guarded(F f) {
  try {
    return f();
  } catch (const Raised &) {
  } catch (const Refused &e) {
    PyErr_SetString(PyExc_ValueError, e.what());
  } catch (const c10::Error &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

// ---------------------------------------------------------------- Pages
struct PagesObject {
  PyObject_HEAD
  PyObject *k, *v;
  locret_pages c;
};
extern PyTypeObject PagesType;

locret_pages described(const at::Tensor &k, const at::Tensor &v) {
  if (k.dim() != 4 || k.sizes() != v.sizes() || k.strides() != v.strides() || k.scalar_type() != v.scalar_type() || k.device() != v.device())
    refuse("keys and values must be alike: [n_pages, n_kv_heads, page_size, head_dim]");
  if (dtype_code(k.scalar_type()) < 0 || !k.is_cuda() || k.stride(3) != 1)
    refuse("pages must be CUDA bfloat16 or float16 tensors, contiguous in the last dimension");
  for (int i = 0; i < 4; i++)
    if (k.size(i) > INT32_MAX) refuse("pages: a size does not fit 32 bits");
  return {k.data_ptr(), v.data_ptr(), (int32_t)k.size(0), (int32_t)k.size(2), (int32_t)k.size(1), (int32_t)k.size(3),
          dtype_code(k.scalar_type()), k.stride(0), k.stride(1), k.stride(2)};
}
// The struct as the tensors are now: a storage may have been replaced since the last call.
const locret_pages &refreshed(PagesObject *p) {
  return p->c = described(THPVariable_Unpack(p->k), THPVariable_Unpack(p->v));
}

PyObject *pages_new(PyTypeObject *type, PyObject *args, PyObject *kwargs) {
  return guarded([&]() -> PyObject * {
    static const char *names[] = {"k", "v", nullptr};
    PyObject *ko, *vo;
    if (!PyArg_ParseTupleAndKeywords(args, kwargs, "OO:Pages", const_cast<char **>(names), &ko, &vo)) throw Raised();
    const locret_pages c = described(tensor(ko, "k"), tensor(vo, "v"));
    PagesObject *self = reinterpret_cast<PagesObject *>(type->tp_alloc(type, 0));
    if (!self) throw Raised();
    Py_INCREF(ko);
    Py_INCREF(vo);
    self->k = ko;
    self->v = vo;
    self->c = c;
    return reinterpret_cast<PyObject *>(self);
  });
}
void pages_dealloc(PyObject *o) {
  PagesObject *self = reinterpret_cast<PagesObject *>(o);
  Py_XDECREF(self->k);
  Py_XDECREF(self->v);
  Py_TYPE(o)->tp_free(o);
}
PyObject *pages_address(PyObject *o, void *) {
  return guarded([&]() -> PyObject * {
    return PyLong_FromVoidPtr(const_cast<locret_pages *>(&refreshed(reinterpret_cast<PagesObject *>(o))));
  });
}

PyMemberDef pages_members[] = {{"k", T_OBJECT_EX, offsetof(PagesObject, k), READONLY, "the keys' tensor"},
                               {"v", T_OBJECT_EX, offsetof(PagesObject, v), READONLY, "the values' tensor"},
                               {nullptr, 0, 0, 0, nullptr}};
PyGetSetDef pages_getset[] = {{"address", pages_address, nullptr, "address of the C struct locret_pages as the tensors are now, for the C entry points", nullptr},
                              {nullptr, nullptr, nullptr, nullptr, nullptr}};
PyTypeObject PagesType = {PyVarObject_HEAD_INIT(nullptr, 0)};

void changed_pages(PyObject *o) {
  changed(reinterpret_cast<PagesObject *>(o)->k);
  changed(reinterpret_cast<PagesObject *>(o)->v);
}
const locret_pages &pages_of(PyObject *o, const Where &w) {
  if (!PyObject_TypeCheck(o, &PagesType)) {
    PyErr_SetString(PyExc_TypeError, "pages must be a Pages");
    throw Raised();
  }
  PagesObject *p = reinterpret_cast<PagesObject *>(o);
  const at::Tensor &k = THPVariable_Unpack(p->k), &v = THPVariable_Unpack(p->v);
  if (k.device() != w.device) refuse("pages must lie on " + w.device.str());
  no_graph(k, "the pages' k");
  no_graph(v, "the pages' v");
  return refreshed(p);
}

// ---------------------------------------------------------------- pages_step
PyTypeObject *step_type = nullptr;
PyStructSequence_Field step_fields[] = {{"slots", "int64 [n_tok]: page * page_size + offset, -1 where a row has no place"},
                                        {"positions", "int32 [n_tok]"},
                                        {"starts", "int32 [n_req + 1]: first row of every request"},
                                        {"lens", "int32 [n_req]: lengths after the step"},
                                        {"n_free", "int32 [1]: pages left on the list"},
                                        {nullptr, nullptr}};
PyStructSequence_Desc step_desc = {"paper_2410_01805_b200.PagesStep", "What a step's bookkeeping made (pages_step).", step_fields, 5};

PyObject *pages_step(PyObject *, PyObject *const *argv, Py_ssize_t n, PyObject *kwnames) {
  return guarded([&]() -> PyObject * {
    static const Names<10> names({"table", "lens", "new_lens", "free_pages", "n_free", "page_size", "n_tok", "lens_out", "n_free_out", "status"});
    const Args<10> a("pages_step", names, 7, argv, n, kwnames);
    const at::Tensor &table = tensor(a.v[0], "table");
    const Where w(table, "table");
    words(a.v[0], "table", at::kInt, 2, w);
    const at::Tensor *lens, *grow, *free_pages, *n_free, *t;
    PyObject *const lens_out = a.v[7] ? a.v[7] : a.v[1], *const n_free_out = a.v[8] ? a.v[8] : a.v[4];
    const int64_t n_req = table.size(0), n_tok = integer(a.v[6], 0);
    void *const lens_p = words(a.v[1], "lens", at::kInt, 1, w, &lens), *const new_p = words(a.v[2], "new_lens", at::kInt, 1, w, &grow),
               *const free_p = words(a.v[3], "free_pages", at::kInt, 1, w, &free_pages),
               *const nf_p = words(a.v[4], "n_free", at::kInt, 1, w, &n_free);
    if (lens->numel() != n_req || grow->numel() != n_req || n_free->numel() != 1)
      refuse("one length and one number of new tokens for every row of the table, and one n_free");
    void *const lens_out_p = words(lens_out, "lens_out", at::kInt, 1, w, &t);
    if (t->numel() != n_req) refuse("lens_out must have the size of lens");
    void *const nf_out_p = words(n_free_out, "n_free_out", at::kInt, 1, w, &t);
    if (t->numel() != 1) refuse("n_free_out must have one element");
    if (n_tok < 0 || n_tok > INT32_MAX || n_req > INT32_MAX || free_pages->numel() > INT32_MAX || table.size(1) > INT32_MAX)
      refuse("n_tok, or the size of a tensor, is out of range");
    at::Tensor slots = empty({n_tok}, at::kLong, w), positions = empty({n_tok}, at::kInt, w), starts = empty({n_req + 1}, at::kInt, w);
    check(locret_pages_step(static_cast<int32_t *>(table.data_ptr()), table.stride(0), (int32_t)table.size(1),
                            static_cast<int32_t *>(lens_p), static_cast<int32_t *>(lens_out_p), static_cast<int32_t *>(new_p),
                            (int32_t)n_req, integer32(a.v[5], 0, "page_size"), static_cast<int32_t *>(free_p),
                            (int32_t)free_pages->numel(), static_cast<int32_t *>(nf_p), static_cast<int32_t *>(nf_out_p),
                            (int32_t)n_tok, static_cast<int64_t *>(slots.data_ptr()), static_cast<int32_t *>(positions.data_ptr()),
                            static_cast<int32_t *>(starts.data_ptr()), status_word(a.v[9], w), w.stream),
          "locret_pages_step");
    for (PyObject *o : {a.v[0], a.v[3], lens_out, n_free_out, a.v[9]}) changed(o);
    PyObject *r = PyStructSequence_New(step_type);
    if (!r) throw Raised();
    Py_INCREF(lens_out);
    Py_INCREF(n_free_out);
    PyStructSequence_SetItem(r, 0, wrap(std::move(slots)));
    PyStructSequence_SetItem(r, 1, wrap(std::move(positions)));
    PyStructSequence_SetItem(r, 2, wrap(std::move(starts)));
    PyStructSequence_SetItem(r, 3, lens_out);
    PyStructSequence_SetItem(r, 4, n_free_out);
    return r;
  });
}

// ---------------------------------------------------------------- norm_rope
void gain(const void *&to, PyObject *o, const char *what, int64_t d, at::ScalarType type, const Where &w) {
  if (!o) return;
  const at::Tensor &g = tensor(o, what);
  if (g.dim() != 1 || g.size(0) != d || g.scalar_type() != type || g.device() != w.device || !g.is_contiguous())
    refuse(std::string(what) + " must be a contiguous vector of " + std::to_string(d) + " elements of type " + c10::toString(type));
  to = g.data_ptr();
}
// what both directions share: y (outputs, or their gradients), positions, turns, gains
void rope_common(locret_rope_args &r, const at::Tensor &yq, int64_t k_heads, PyObject *positions, PyObject *turns, PyObject *factor,
                 PyObject *interleaved, PyObject *g_q, PyObject *g_k, PyObject *eps, const Where &w) {
  const at::Tensor *t;
  r.positions = static_cast<int32_t *>(words(positions, "positions", at::kInt, 1, w, &t));
  if (t->numel() != yq.size(0)) refuse("one position for every token");
  r.turns = static_cast<uint64_t *>(words(turns, "turns", at::kLong, 1, w, &t));
  if (t->numel() > 1 << 20 || yq.size(0) > INT32_MAX || yq.size(1) > INT32_MAX || yq.size(2) > INT32_MAX || k_heads > INT32_MAX)
    refuse("a size does not fit 32 bits");
  r.rot = 2 * (int32_t)t->numel();
  r.n_tok = (int32_t)yq.size(0);
  r.n_q_heads = (int32_t)yq.size(1);
  r.n_kv_heads = (int32_t)k_heads;
  r.head_dim = (int32_t)yq.size(2);
  r.dtype = dtype_code(yq.scalar_type());
  r.factor = (float)number(factor, 1.0);
  r.interleaved = truth(interleaved);
  r.eps = (float)number(eps, 1e-6);
  gain(r.g_q, g_q, "g_q", yq.size(2), yq.scalar_type(), w);
  gain(r.g_k, g_k, "g_k", yq.size(2), yq.scalar_type(), w);
}
void input(const void *&p, int64_t &token, int64_t &head, const at::Tensor &t) { p = t.data_ptr(); token = t.stride(0); head = t.stride(1); }
void output(void *&p, int64_t &token, int64_t &head, const at::Tensor &t) { p = t.data_ptr(); token = t.stride(0); head = t.stride(1); }

PyObject *norm_rope(PyObject *, PyObject *const *argv, Py_ssize_t n, PyObject *kwnames) {
  return guarded([&]() -> PyObject * {
    static const Names<15> names({"q", "k", "positions", "turns", "factor", "interleaved", "g_q", "g_k", "eps", "q_out", "k_out", "v", "pages", "slots", "status"});
    const Args<15> a("norm_rope", names, 4, argv, n, kwnames);
    const at::Tensor &q0 = tensor(a.v[0], "q");
    const Where w(q0, "q");
    const at::ScalarType type = q0.scalar_type();
    const at::Tensor &q = heads(a.v[0], "q", type, w), &k = heads(a.v[1], "k", type, w);
    no_graph(q, "q");
    no_graph(k, "k");
    if (k.size(0) != q.size(0) || k.size(2) != q.size(2)) refuse("q and k must have the same tokens and head size");
    if (!a.v[12] != !a.v[11] || !a.v[12] != !a.v[13]) refuse("pages, v and slots come together");
    locret_rope_args r = {};
    input(r.q, r.q_token, r.q_head, q);
    input(r.k, r.k_token, r.k_head, k);
    at::Tensor q_out, k_out;
    if (a.v[9]) q_out = written(a.v[9], "q_out", type, w);
    if (a.v[10]) k_out = written(a.v[10], "k_out", type, w);
    if (a.v[12]) {
      const at::Tensor &v = heads(a.v[11], "v", type, w), *slots;
      same_shape(v, k, "v and k");
      no_graph(v, "v");
      input(r.v, r.v_token, r.v_head, v);
      r.pages = &pages_of(a.v[12], w);
      r.slots = static_cast<int64_t *>(words(a.v[13], "slots", at::kLong, 1, w, &slots));
      if (slots->numel() != q.size(0)) refuse("one slot for every token");
    }
    if (a.v[6]) no_graph(tensor(a.v[6], "g_q"), "g_q");
    if (a.v[7]) no_graph(tensor(a.v[7], "g_k"), "g_k");
    rope_common(r, q, k.size(1), a.v[2], a.v[3], a.v[4], a.v[5], a.v[6], a.v[7], a.v[8], w);
    r.status = status_word(a.v[14], w);
    if (!a.v[9]) q_out = empty(q.sizes(), type, w);
    if (!a.v[10] && !a.v[12]) k_out = empty(k.sizes(), type, w);
    same_shape(q_out, q, "q_out and q");
    output(r.q_out, r.q_out_token, r.q_out_head, q_out);
    if (k_out.defined()) {
      same_shape(k_out, k, "k_out and k");
      output(r.k_out, r.k_out_token, r.k_out_head, k_out);
    }
    check(locret_norm_rope(&r, w.stream), "locret_norm_rope");
    for (PyObject *o : {a.v[9], a.v[10], a.v[14]}) changed(o);
    if (a.v[12]) changed_pages(a.v[12]);
    PyObject *qo = wrap(std::move(q_out)), *ko = k_out.defined() ? wrap(std::move(k_out)) : Py_NewRef(Py_None);
    PyObject *res = PyTuple_Pack(2, qo, ko);
    Py_DECREF(qo);
    Py_DECREF(ko);
    return res;
  });
}

PyObject *norm_rope_grad(PyObject *, PyObject *const *argv, Py_ssize_t n, PyObject *kwnames) {
  return guarded([&]() -> PyObject * {
    static const Names<11> names({"dq_out", "dk_out", "q", "k", "positions", "turns", "factor", "interleaved", "g_q", "g_k", "eps"});
    const Args<11> a("norm_rope_grad", names, 2, argv, n, kwnames);
    const at::Tensor &dq0 = tensor(a.v[0], "dq_out");
    const Where w(dq0, "dq_out");
    const at::ScalarType type = dq0.scalar_type();
    const at::Tensor &dq_out = heads(a.v[0], "dq_out", type, w), &dk_out = heads(a.v[1], "dk_out", type, w);
    if (dk_out.size(0) != dq_out.size(0) || dk_out.size(2) != dq_out.size(2)) refuse("dq_out and dk_out must have the same tokens and head size");
    if (!a.v[4] || !a.v[5]) Args<11>::fail("norm_rope_grad", "needs 'positions' and 'turns'");
    if ((a.v[8] && !a.v[2]) || (a.v[9] && !a.v[3])) refuse("q and k must be the forward call's inputs where there is a norm");
    locret_rope_args r = {};
    if (a.v[2]) {
      const at::Tensor &q = heads(a.v[2], "q", type, w);
      same_shape(q, dq_out, "q and dq_out");
      input(r.q, r.q_token, r.q_head, q);
    }
    if (a.v[3]) {
      const at::Tensor &k = heads(a.v[3], "k", type, w);
      same_shape(k, dk_out, "k and dk_out");
      input(r.k, r.k_token, r.k_head, k);
    }
    output(r.q_out, r.q_out_token, r.q_out_head, dq_out);
    output(r.k_out, r.k_out_token, r.k_out_head, dk_out);
    rope_common(r, dq_out, dk_out.size(1), a.v[4], a.v[5], a.v[6], a.v[7], a.v[8], a.v[9], a.v[10], w);
    const int64_t d = dq_out.size(2);
    at::Tensor dq = empty(dq_out.sizes(), type, w), dk = empty(dk_out.sizes(), type, w), dg_q, dg_k, ws;
    if (r.g_q) dg_q = empty({d}, at::kFloat, w);
    if (r.g_k) dg_k = empty({d}, at::kFloat, w);
    int64_t need = 0;
    if (r.g_q || r.g_k) {
      check(locret_norm_rope_grad_workspace((int32_t)d, &need), "locret_norm_rope_grad");
      ws = empty({need}, at::kByte, w);
    }
    check(locret_norm_rope_grad(&r, dq.data_ptr(), dk.data_ptr(), dg_q.defined() ? static_cast<float *>(dg_q.data_ptr()) : nullptr,
                                dg_k.defined() ? static_cast<float *>(dg_k.data_ptr()) : nullptr,
                                ws.defined() ? ws.data_ptr() : nullptr, need, w.stream),
          "locret_norm_rope_grad");
    PyObject *o[4] = {wrap(std::move(dq)), wrap(std::move(dk)), dg_q.defined() ? wrap(std::move(dg_q)) : Py_NewRef(Py_None),
                      dg_k.defined() ? wrap(std::move(dg_k)) : Py_NewRef(Py_None)};
    PyObject *res = PyTuple_Pack(4, o[0], o[1], o[2], o[3]);
    for (PyObject *x : o) Py_DECREF(x);
    return res;
  });
}

// ---------------------------------------------------------------- paged_attention
PyObject *paged_attention(PyObject *, PyObject *const *argv, Py_ssize_t n, PyObject *kwnames) {
  return guarded([&]() -> PyObject * {
    static const Names<10> names({"q", "pages", "table", "lens", "scale", "window", "sinks", "out", "with_lse", "status"});
    const Args<10> a("paged_attention", names, 4, argv, n, kwnames);
    const at::Tensor &q0 = tensor(a.v[0], "q");
    const Where w(q0, "q");
    const locret_pages &pages = pages_of(a.v[1], w);
    const at::Tensor &q = heads(a.v[0], "q", q0.scalar_type(), w), *table, *lens;
    no_graph(q, "q");
    if (dtype_code(q.scalar_type()) != pages.dtype || q.size(2) != pages.head_dim) refuse("q must have the pages' type and head size");
    void *const table_p = words(a.v[2], "table", at::kInt, 2, w, &table), *const lens_p = words(a.v[3], "lens", at::kInt, 1, w, &lens);
    if (table->size(0) != q.size(0) || lens->numel() != q.size(0)) refuse("one row of the table and one length for every request");
    if (q.size(0) > INT32_MAX || q.size(1) > INT32_MAX || table->size(1) > INT32_MAX) refuse("a size does not fit 32 bits");
    const int32_t h = (int32_t)q.size(1);
    at::Tensor out, lse;
    if (a.v[7]) {
      out = written(a.v[7], "out", q.scalar_type(), w);
      same_shape(out, q, "out and q");
    } else {
      out = empty(q.sizes(), q.scalar_type(), w);
    }
    if (truth(a.v[8])) lse = empty({q.size(0), q.size(1)}, at::kFloat, w);
    int64_t need = 0;
    check(locret_paged_attention_workspace(h, pages.n_kv_heads, pages.head_dim, &need), "locret_paged_attention");
    at::Tensor ws = empty({need}, at::kByte, w);
    check(locret_paged_attention(q.data_ptr(), q.stride(0), q.stride(1), &pages, static_cast<int32_t *>(table_p), table->stride(0),
                                 (int32_t)table->size(1), static_cast<int32_t *>(lens_p), (int32_t)q.size(0), h,
                                 (float)number(a.v[4], 1.0 / std::sqrt((double)pages.head_dim)), integer32(a.v[5], 0, "window"),
                                 integer32(a.v[6], 0, "sinks"), out.data_ptr(), out.stride(0), out.stride(1),
                                 lse.defined() ? static_cast<float *>(lse.data_ptr()) : nullptr, status_word(a.v[9], w),
                                 ws.data_ptr(), need, w.stream),
          "locret_paged_attention");
    for (PyObject *o : {a.v[7], a.v[9]}) changed(o);
    if (!lse.defined()) return wrap(std::move(out));
    PyObject *o = wrap(std::move(out)), *l = wrap(std::move(lse)), *res = PyTuple_Pack(2, o, l);
    Py_DECREF(o);
    Py_DECREF(l);
    return res;
  });
}

#define METHOD(f, doc) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL | METH_KEYWORDS, doc}
PyMethodDef methods[] = {
    METHOD(pages_step,
           "pages_step(table, lens, new_lens, free_pages, n_free, page_size, n_tok, lens_out=None, n_free_out=None, status=None)\n--\n\n"
           "One step's bookkeeping: table int32 [n_req, width], lens, new_lens int32 [n_req] (new_lens < 0: the request has ended),\n"
           "free_pages int32 [number of pages], n_free int32 [1].  table and free_pages are updated in place, lens and n_free too\n"
           "unless lens_out and n_free_out are given.  Returns a PagesStep of n_tok rows."),
    METHOD(norm_rope,
           "norm_rope(q, k, positions, turns, factor=1.0, interleaved=False, g_q=None, g_k=None, eps=1e-6, q_out=None, k_out=None,\n"
           "          v=None, pages=None, slots=None, status=None)\n--\n\n"
           "Per-head RMS norm (with gains g_q, g_k, if given), rotation at `positions` (int32 [n_tok]) and, with pages, the rotated\n"
           "keys and the values v into `slots` (int64 [n_tok], negative: none): q [n_tok, h, d], k and v [n_tok, h_kv, d], bf16 or\n"
           "fp16, of any token and head strides -> (q_out, k_out).  Outputs are allocated where none are given, k_out only without\n"
           "pages; q_out may be q and k_out k.  turns, factor: of rope_turns.  Not recorded for autograd: inputs that require gradients\n"
           "are refused unless recording is off, as in the forward of a torch.autograd.Function (norm_rope_grad in its backward)."),
    METHOD(norm_rope_grad,
           "norm_rope_grad(dq_out, dk_out, q, k, positions, turns, factor=1.0, interleaved=False, g_q=None, g_k=None, eps=1e-6)\n--\n\n"
           "Gradients of norm_rope from those of its outputs: (dq, dk, dg_q, dg_k), the latter fp32 [d] where a gain is given and\n"
           "None elsewhere.  q and k are the inputs of the forward call, needed where there is a gain."),
    METHOD(paged_attention,
           "paged_attention(q, pages, table, lens, scale=None, window=0, sinks=0, out=None, with_lse=False, status=None)\n--\n\n"
           "Attention of each request's newest token, q [n_req, h, d], over the keys and values in its pages: table int32\n"
           "[n_req, width], lens int32 [n_req] (the new token counted).  window > 0: only the last `window` and the first `sinks`\n"
           "tokens are visible.  scale: 1 / sqrt(d) by default.  Returns out, [n_req, h, d], or (out, lse fp32 [n_req, h]).  There is no\n"
           "backward pass: inputs that require gradients are refused unless recording is off."),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", "Python entry points of the calls on pages (" BUILT_FOR ").", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged() {
  PagesType.tp_name = "paper_2410_01805_b200.Pages";
  PagesType.tp_basicsize = sizeof(PagesObject);
  PagesType.tp_flags = Py_TPFLAGS_DEFAULT;
  PagesType.tp_doc = "Pages(k, v)\n--\n\nOne layer's pool: keys and values [n_pages, n_kv_heads, page_size, head_dim], bf16 or fp16, views of any layout\n"
                     "(the same for both) whose last dimension is contiguous.";
  PagesType.tp_new = pages_new;
  PagesType.tp_dealloc = pages_dealloc;
  PagesType.tp_members = pages_members;
  PagesType.tp_getset = pages_getset;
  if (PyType_Ready(&PagesType) < 0) return nullptr;
  PyObject *m = PyModule_Create(&module);
  if (!m) return nullptr;
  step_type = PyStructSequence_NewType(&step_desc);
  if (!step_type) return nullptr;
  Py_INCREF(&PagesType);
  PyModule_AddObject(m, "Pages", reinterpret_cast<PyObject *>(&PagesType));
  PyModule_AddObject(m, "PagesStep", reinterpret_cast<PyObject *>(step_type));
  module_self = m;
  return m;
}
