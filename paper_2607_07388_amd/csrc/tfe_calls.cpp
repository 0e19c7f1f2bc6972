// The per-step calls of the Python binding (lookups, prefetches, head top-K,
// the calls on logits) as functions of a CPython module: a decode step's launch is a few
// microseconds, of which marshalling its arguments through ctypes took about
// half.  Each function takes the plain case -- positional arguments, exact
// ints, floats and None, objects with data_ptr() -- and hands everything else
// to the ctypes function of the same name, whose conversions and errors
// apply.  The library's functions are bound by address, so this module links
// with nothing.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

namespace {

PyObject* g_check;         // raises for a negative status
PyObject* g_data_ptr;      // "data_ptr"
PyObject* g_cuda_stream;   // "cuda_stream"

struct Call {
  PyObject* slow;  // the ctypes function
  void* fn;
};
Call g_lookup, g_multi, g_prefetch, g_scored, g_topk, g_linear, g_sample, g_loss, g_grad, g_both;
Call g_xent, g_xent_grad, g_xent_both, g_norm, g_clip, g_norm_clip, g_int8;

// Each conversion returns false, with no exception set, for what the plain
// case does not cover.
bool from_int(PyObject* o, void** out) {
  if (!PyLong_CheckExact(o)) return false;
  *out = PyLong_AsVoidPtr(o);
  if (*out == nullptr && PyErr_Occurred()) {
    PyErr_Clear();
    return false;
  }
  return true;
}
bool handle(PyObject* o, void** out) {
  *out = nullptr;
  return o == Py_None || from_int(o, out);
}
bool pointer(PyObject* o, void** out) {
  if (handle(o, out)) return true;
  if (PyLong_Check(o)) return false;
  PyObject* r = PyObject_CallMethodNoArgs(o, g_data_ptr);
  if (!r) {
    PyErr_Clear();
    return false;
  }
  const bool ok = from_int(r, out);
  Py_DECREF(r);
  return ok;
}
bool stream(PyObject* o, void** out) {
  if (handle(o, out)) return true;
  if (PyLong_Check(o)) return false;
  PyObject* r = PyObject_GetAttr(o, g_cuda_stream);
  if (!r) {
    PyErr_Clear();
    return false;
  }
  const bool ok = from_int(r, out);
  Py_DECREF(r);
  return ok;
}
bool int32(PyObject* o, int32_t* out) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if (over || v < INT32_MIN || v > INT32_MAX) return false;
  *out = (int32_t)v;
  return true;
}
bool int64(PyObject* o, int64_t* out) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long long v = PyLong_AsLongLongAndOverflow(o, &over);
  if (over) return false;
  *out = (int64_t)v;
  return true;
}
bool number(PyObject* o, float* out) {
  if (!PyFloat_CheckExact(o)) return false;
  *out = (float)PyFloat_AS_DOUBLE(o);
  return true;
}

PyObject* slow(const Call& c, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  return PyObject_Vectorcall(c.slow, a, (size_t)n, kw);
}
PyObject* status(int st) {
  if (st < 0) return PyObject_CallFunction(g_check, "i", st);
  return PyLong_FromLong(st);
}

#define SLOW_UNLESS(c, cond) \
  if (!(cond)) return slow(c, a, n, kw)
// Arguments [0, need) and an optional stream behind them.
#define PLAIN(c, need) \
  void* s = nullptr;   \
  SLOW_UNLESS(c, !kw && (n == (need) || (n == (need) + 1 && stream(a[need], &s))))

PyObject* lookup_inject(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_lookup, 12);
  void *t, *tok, *hin, *hout, *hit, *slot, *len;
  int32_t B, ctx, S, gate;
  float scale;
  SLOW_UNLESS(g_lookup, handle(a[0], &t) && pointer(a[1], &tok) && int32(a[2], &B) &&
                            int32(a[3], &ctx) && int32(a[4], &S) && pointer(a[5], &hin) &&
                            pointer(a[6], &hout) && pointer(a[7], &hit) && pointer(a[8], &slot) &&
                            pointer(a[9], &len) && int32(a[10], &gate) && number(a[11], &scale));
  using Fn = int (*)(void*, void*, int32_t, int32_t, int32_t, void*, void*, void*, void*, void*,
                     int32_t, float, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_lookup.fn)(t, tok, B, ctx, S, hin, hout, hit, slot, len, gate, scale, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* lookup_inject_multi(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_multi, 12);
  void *t, *tok, *hin, *hout, *mask, *slot;
  int32_t B, ctx, S, weighting, gate;
  float scale;
  SLOW_UNLESS(g_multi, handle(a[0], &t) && pointer(a[1], &tok) && int32(a[2], &B) &&
                           int32(a[3], &ctx) && int32(a[4], &S) && pointer(a[5], &hin) &&
                           pointer(a[6], &hout) && pointer(a[7], &mask) && pointer(a[8], &slot) &&
                           int32(a[9], &weighting) && int32(a[10], &gate) && number(a[11], &scale));
  using Fn = int (*)(void*, void*, int32_t, int32_t, int32_t, void*, void*, void*, void*, int32_t,
                     int32_t, float, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_multi.fn)(t, tok, B, ctx, S, hin, hout, mask, slot, weighting, gate, scale, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* prefetch(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_prefetch, 6);
  void *t, *tail, *cand;
  int32_t tl, B, K;
  SLOW_UNLESS(g_prefetch, handle(a[0], &t) && pointer(a[1], &tail) && int32(a[2], &tl) &&
                              pointer(a[3], &cand) && int32(a[4], &B) && int32(a[5], &K));
  using Fn = int (*)(void*, void*, int32_t, void*, int32_t, int32_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_prefetch.fn)(t, tail, tl, cand, B, K, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* prefetch_scored(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_scored, 8);
  void *t, *tail, *cand, *prob;
  int32_t tl, B, K, budget;
  SLOW_UNLESS(g_scored, handle(a[0], &t) && pointer(a[1], &tail) && int32(a[2], &tl) &&
                            pointer(a[3], &cand) && pointer(a[4], &prob) && int32(a[5], &B) &&
                            int32(a[6], &K) && int32(a[7], &budget));
  using Fn = int (*)(void*, void*, int32_t, void*, void*, int32_t, int32_t, int32_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_scored.fn)(t, tail, tl, cand, prob, B, K, budget, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* head_topk(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_topk, 6);
  void *h, *hid, *ids, *prob;
  int32_t B, K;
  SLOW_UNLESS(g_topk, handle(a[0], &h) && pointer(a[1], &hid) && int32(a[2], &B) &&
                          int32(a[3], &K) && pointer(a[4], &ids) && pointer(a[5], &prob));
  using Fn = int (*)(void*, void*, int32_t, int32_t, void*, void*, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_topk.fn)(h, hid, B, K, ids, prob, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* quantized_linear(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_linear, 13);
  void *x, *w, *ws, *out, *space;
  int64_t ldx, rows, ldo, bytes;
  int32_t dtype, odt, od, dim;
  SLOW_UNLESS(g_linear, pointer(a[0], &x) && int32(a[1], &dtype) && int64(a[2], &ldx) &&
                            pointer(a[3], &w) && pointer(a[4], &ws) && int64(a[5], &rows) &&
                            int32(a[6], &od) && int32(a[7], &dim) && pointer(a[8], &out) &&
                            int32(a[9], &odt) && int64(a[10], &ldo) && pointer(a[11], &space) &&
                            int64(a[12], &bytes));
  using Fn = int (*)(void*, int32_t, int64_t, void*, void*, int64_t, int32_t, int32_t, void*,
                     int32_t, int64_t, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_linear.fn)(x, dtype, ldx, w, ws, rows, od, dim, out, odt, ldo, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_sample, 14);
  void *l, *T, *k, *p, *m, *u, *token, *prob, *space;
  int64_t ld, rows, bytes;
  int32_t dtype, vocab;
  SLOW_UNLESS(g_sample, pointer(a[0], &l) && int32(a[1], &dtype) && int64(a[2], &ld) &&
                            int64(a[3], &rows) && int32(a[4], &vocab) && pointer(a[5], &T) &&
                            pointer(a[6], &k) && pointer(a[7], &p) && pointer(a[8], &m) &&
                            pointer(a[9], &u) && pointer(a[10], &token) && pointer(a[11], &prob) &&
                            pointer(a[12], &space) && int64(a[13], &bytes));
  using Fn = int (*)(void*, int32_t, int64_t, int64_t, int32_t, void*, void*, void*, void*, void*,
                     void*, void*, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_sample.fn)(l, dtype, ld, rows, vocab, T, k, p, m, u, token, prob, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

// What the three distillation calls begin with.
struct Distill {
  void *l, *ids, *t;
  int64_t ld, rows;
  int32_t dtype, vocab, tdtype, K;
  float tau;
};
bool distill(PyObject* const* a, Distill* d) {
  return pointer(a[0], &d->l) && int32(a[1], &d->dtype) && int64(a[2], &d->ld) &&
         int64(a[3], &d->rows) && int32(a[4], &d->vocab) && pointer(a[5], &d->ids) &&
         pointer(a[6], &d->t) && int32(a[7], &d->tdtype) && int32(a[8], &d->K) &&
         number(a[9], &d->tau);
}

PyObject* distill_loss(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_loss, 14);
  Distill d;
  void *loss, *lse, *space;
  int64_t bytes;
  SLOW_UNLESS(g_loss, distill(a, &d) && pointer(a[10], &loss) && pointer(a[11], &lse) &&
                          pointer(a[12], &space) && int64(a[13], &bytes));
  using Fn = int (*)(void*, int32_t, int64_t, int64_t, int32_t, void*, void*, int32_t, int32_t,
                     float, void*, void*, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_loss.fn)(d.l, d.dtype, d.ld, d.rows, d.vocab, d.ids, d.t, d.tdtype, d.K, d.tau, loss,
                       lse, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* distill_grad(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_grad, 14);
  Distill d;
  void *lse, *weight, *grad;
  int64_t ldg;
  SLOW_UNLESS(g_grad, distill(a, &d) && pointer(a[10], &lse) && pointer(a[11], &weight) &&
                          pointer(a[12], &grad) && int64(a[13], &ldg));
  using Fn = int (*)(void*, int32_t, int64_t, int64_t, int32_t, void*, void*, int32_t, int32_t,
                     float, void*, void*, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_grad.fn)(d.l, d.dtype, d.ld, d.rows, d.vocab, d.ids, d.t, d.tdtype, d.K, d.tau, lse,
                       weight, grad, ldg, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* distill_loss_grad(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_both, 17);
  Distill d;
  void *weight, *loss, *lse, *grad, *space;
  int64_t ldg, bytes;
  SLOW_UNLESS(g_both, distill(a, &d) && pointer(a[10], &weight) && pointer(a[11], &loss) &&
                          pointer(a[12], &lse) && pointer(a[13], &grad) && int64(a[14], &ldg) &&
                          pointer(a[15], &space) && int64(a[16], &bytes));
  using Fn = int (*)(void*, int32_t, int64_t, int64_t, int32_t, void*, void*, int32_t, int32_t,
                     float, void*, void*, void*, void*, int64_t, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_both.fn)(d.l, d.dtype, d.ld, d.rows, d.vocab, d.ids, d.t, d.tdtype, d.K, d.tau,
                       weight, loss, lse, grad, ldg, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* integer_linear(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_int8, 13);
  void *x, *w, *ws, *out, *space;
  int64_t ldx, rows, ldo, bytes;
  int32_t dtype, odt, od, dim;
  SLOW_UNLESS(g_int8, pointer(a[0], &x) && int32(a[1], &dtype) && int64(a[2], &ldx) &&
                            pointer(a[3], &w) && pointer(a[4], &ws) && int64(a[5], &rows) &&
                            int32(a[6], &od) && int32(a[7], &dim) && pointer(a[8], &out) &&
                            int32(a[9], &odt) && int64(a[10], &ldo) && pointer(a[11], &space) &&
                            int64(a[12], &bytes));
  using Fn = int (*)(void*, int32_t, int64_t, void*, void*, int64_t, int32_t, int32_t, void*,
                     int32_t, int64_t, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_int8.fn)(x, dtype, ldx, w, ws, rows, od, dim, out, odt, ldo, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

// The arguments that the cross entropy calls begin with.
struct Xent {
  void *h, *w, *t;
  int64_t ldh, ldw, rows;
  int32_t vocab, dim;
};
bool xent(PyObject* const* a, Xent* x) {
  return pointer(a[0], &x->h) && int64(a[1], &x->ldh) && pointer(a[2], &x->w) &&
         int64(a[3], &x->ldw) && pointer(a[4], &x->t) && int64(a[5], &x->rows) &&
         int32(a[6], &x->vocab) && int32(a[7], &x->dim);
}
// Gradients and workspace, from a on.
struct XentGrads {
  void *gx, *gw, *space;
  int64_t ldgx, ldgw, bytes;
  int32_t dtype, add;
};
bool xent_grads(PyObject* const* a, XentGrads* g) {
  return pointer(a[0], &g->gx) && int64(a[1], &g->ldgx) && pointer(a[2], &g->gw) &&
         int64(a[3], &g->ldgw) && int32(a[4], &g->dtype) && int32(a[5], &g->add) &&
         pointer(a[6], &g->space) && int64(a[7], &g->bytes);
}

PyObject* cross_entropy_loss(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_xent, 12);
  Xent x;
  void *loss, *lse, *space;
  int64_t bytes;
  SLOW_UNLESS(g_xent, xent(a, &x) && pointer(a[8], &loss) && pointer(a[9], &lse) &&
                          pointer(a[10], &space) && int64(a[11], &bytes));
  using Fn = int (*)(void*, int64_t, void*, int64_t, void*, int64_t, int32_t, int32_t, void*, void*,
                     void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_xent.fn)(x.h, x.ldh, x.w, x.ldw, x.t, x.rows, x.vocab, x.dim, loss, lse, space, bytes,
                       s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* cross_entropy_grad(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_xent_grad, 18);
  Xent x;
  XentGrads g;
  void *lse, *weight;
  SLOW_UNLESS(g_xent_grad, xent(a, &x) && pointer(a[8], &lse) && pointer(a[9], &weight) &&
                               xent_grads(a + 10, &g));
  using Fn = int (*)(void*, int64_t, void*, int64_t, void*, int64_t, int32_t, int32_t, void*, void*,
                     void*, int64_t, void*, int64_t, int32_t, int32_t, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_xent_grad.fn)(x.h, x.ldh, x.w, x.ldw, x.t, x.rows, x.vocab, x.dim, lse, weight, g.gx,
                            g.ldgx, g.gw, g.ldgw, g.dtype, g.add, g.space, g.bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* cross_entropy_loss_grad(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_xent_both, 19);
  Xent x;
  XentGrads g;
  void *weight, *loss, *lse;
  SLOW_UNLESS(g_xent_both, xent(a, &x) && pointer(a[8], &weight) && pointer(a[9], &loss) &&
                               pointer(a[10], &lse) && xent_grads(a + 11, &g));
  using Fn = int (*)(void*, int64_t, void*, int64_t, void*, int64_t, int32_t, int32_t, void*, void*,
                     void*, void*, int64_t, void*, int64_t, int32_t, int32_t, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_xent_both.fn)(x.h, x.ldh, x.w, x.ldw, x.t, x.rows, x.vocab, x.dim, weight, loss, lse,
                            g.gx, g.ldgx, g.gw, g.ldgw, g.dtype, g.add, g.space, g.bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_norm, 5);
  void *list, *norm, *space;
  int64_t count, bytes;
  SLOW_UNLESS(g_norm, pointer(a[0], &list) && int64(a[1], &count) && pointer(a[2], &norm) &&
                          pointer(a[3], &space) && int64(a[4], &bytes));
  using Fn = int (*)(void*, int64_t, void*, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_norm.fn)(list, count, norm, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* grad_clip(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_clip, 4);
  void *list, *norm;
  int64_t count;
  float most;
  SLOW_UNLESS(g_clip, pointer(a[0], &list) && int64(a[1], &count) && number(a[2], &most) &&
                          pointer(a[3], &norm));
  using Fn = int (*)(void*, int64_t, float, void*, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_clip.fn)(list, count, most, norm, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

PyObject* grad_norm_clip(PyObject*, PyObject* const* a, Py_ssize_t n, PyObject* kw) {
  PLAIN(g_norm_clip, 6);
  void *list, *norm, *space;
  int64_t count, bytes;
  float most;
  SLOW_UNLESS(g_norm_clip, pointer(a[0], &list) && int64(a[1], &count) && number(a[2], &most) &&
                               pointer(a[3], &norm) && pointer(a[4], &space) && int64(a[5], &bytes));
  using Fn = int (*)(void*, int64_t, float, void*, void*, int64_t, void*);
  int st;
  Py_BEGIN_ALLOW_THREADS;
  st = ((Fn)g_norm_clip.fn)(list, count, most, norm, space, bytes, s);
  Py_END_ALLOW_THREADS;
  return status(st);
}

// bind(check, {name: (ctypes function wrapper, address)}); of the calls on
// logits any may be left out, and stays as it is.
PyObject* bind(PyObject*, PyObject* args) {
  PyObject *check, *calls;
  if (!PyArg_ParseTuple(args, "OO!", &check, &PyDict_Type, &calls)) return nullptr;
  const struct {
    const char* name;
    Call* c;
    bool optional;
  } all[] = {{"tfe_lookup_inject", &g_lookup, false},
             {"tfe_lookup_inject_multi", &g_multi, false},
             {"tfe_prefetch", &g_prefetch, false},
             {"tfe_prefetch_scored", &g_scored, false},
             {"tfe_head_topk", &g_topk, false},
             {"tfe_quantized_linear", &g_linear, true},
             {"tfe_sample", &g_sample, true},
             {"tfe_distill_loss", &g_loss, true},
             {"tfe_distill_grad", &g_grad, true},
             {"tfe_distill_loss_grad", &g_both, true},
             {"tfe_cross_entropy_loss", &g_xent, true},
             {"tfe_cross_entropy_grad", &g_xent_grad, true},
             {"tfe_cross_entropy_loss_grad", &g_xent_both, true},
             {"tfe_grad_norm", &g_norm, true},
             {"tfe_grad_clip", &g_clip, true},
             {"tfe_grad_norm_clip", &g_norm_clip, true},
             {"tfe_integer_linear", &g_int8, true}};
  for (const auto& e : all) {
    PyObject* v = PyDict_GetItemString(calls, e.name);
    PyObject *f, *p;
    if (!v && e.optional) continue;
    if (!v || !PyArg_ParseTuple(v, "OO", &f, &p)) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_KeyError, e.name);
      return nullptr;
    }
    void* fn = PyLong_AsVoidPtr(p);
    if (!fn) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.name);
      return nullptr;
    }
    Py_INCREF(f);
    Py_XDECREF(e.c->slow);
    e.c->slow = f;
    e.c->fn = fn;
  }
  Py_INCREF(check);
  Py_XDECREF(g_check);
  g_check = check;
  Py_RETURN_NONE;
}

#define FAST METH_FASTCALL | METH_KEYWORDS
PyMethodDef g_methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"tfe_lookup_inject", (PyCFunction)(void (*)(void))lookup_inject, FAST,
     "tfe_lookup_inject($module, table, tokens, B, ctx, S, hidden_in, hidden_out, hit_mask, "
     "slot_ids, match_len, gate, scale, stream=None)\n--\n\n"},
    {"tfe_lookup_inject_multi", (PyCFunction)(void (*)(void))lookup_inject_multi, FAST,
     "tfe_lookup_inject_multi($module, table, tokens, B, ctx, S, hidden_in, hidden_out, "
     "match_mask, slot_ids, weighting, gate, scale, stream=None)\n--\n\n"},
    {"tfe_prefetch", (PyCFunction)(void (*)(void))prefetch, FAST,
     "tfe_prefetch($module, table, tail, tail_len, candidates, B, K, side_stream=None)\n--\n\n"},
    {"tfe_prefetch_scored", (PyCFunction)(void (*)(void))prefetch_scored, FAST,
     "tfe_prefetch_scored($module, table, tail, tail_len, candidates, cand_prob, B, K, budget, "
     "side_stream=None)\n--\n\n"},
    {"tfe_head_topk", (PyCFunction)(void (*)(void))head_topk, FAST,
     "tfe_head_topk($module, head, hidden, B, K, top_ids, top_prob, stream=None)\n--\n\n"},
    {"tfe_quantized_linear", (PyCFunction)(void (*)(void))quantized_linear, FAST,
     "tfe_quantized_linear($module, x, dtype, ldx, w, w_scales, rows, out_dim, dim, out, out_dtype, "
     "ldo, workspace, workspace_bytes, stream=None)\n--\n\n"},
    {"tfe_sample", (PyCFunction)(void (*)(void))sample, FAST,
     "tfe_sample($module, logits, dtype, ld, rows, vocab, temperature, top_k, top_p, min_p, u, "
     "token, prob, workspace, workspace_bytes, stream=None)\n--\n\n"},
    {"tfe_distill_loss", (PyCFunction)(void (*)(void))distill_loss, FAST,
     "tfe_distill_loss($module, logits, dtype, ld, rows, vocab, teacher_ids, teacher_logits, "
     "teacher_dtype, K, temperature, loss, lse, workspace, workspace_bytes, stream=None)\n--\n\n"},
    {"tfe_distill_grad", (PyCFunction)(void (*)(void))distill_grad, FAST,
     "tfe_distill_grad($module, logits, dtype, ld, rows, vocab, teacher_ids, teacher_logits, "
     "teacher_dtype, K, temperature, lse, grad_loss, grad, ldg, stream=None)\n--\n\n"},
    {"tfe_distill_loss_grad", (PyCFunction)(void (*)(void))distill_loss_grad, FAST,
     "tfe_distill_loss_grad($module, logits, dtype, ld, rows, vocab, teacher_ids, teacher_logits, "
     "teacher_dtype, K, temperature, grad_loss, loss, lse, grad, ldg, workspace, workspace_bytes, "
     "stream=None)\n--\n\n"},
    {"tfe_cross_entropy_loss", (PyCFunction)(void (*)(void))cross_entropy_loss, FAST,
     "tfe_cross_entropy_loss($module, hidden, ldh, w, ldw, targets, rows, vocab, dim, loss, "
     "lse, workspace, workspace_bytes, stream=None)\n--\n\n"},
    {"tfe_cross_entropy_grad", (PyCFunction)(void (*)(void))cross_entropy_grad, FAST,
     "tfe_cross_entropy_grad($module, hidden, ldh, w, ldw, targets, rows, vocab, dim, lse, "
     "grad_loss, grad_hidden, ldgh, grad_w, ldgw, grad_dtype, accumulate, workspace, "
     "workspace_bytes, stream=None)\n--\n\n"},
    {"tfe_cross_entropy_loss_grad", (PyCFunction)(void (*)(void))cross_entropy_loss_grad, FAST,
     "tfe_cross_entropy_loss_grad($module, hidden, ldh, w, ldw, targets, rows, vocab, dim, "
     "grad_loss, loss, lse, grad_hidden, ldgh, grad_w, ldgw, grad_dtype, accumulate, "
     "workspace, workspace_bytes, stream=None)\n--\n\n"},
    {"tfe_grad_norm", (PyCFunction)(void (*)(void))grad_norm, FAST,
     "tfe_grad_norm($module, tensors, n, norm, workspace, workspace_bytes, "
     "stream=None)\n--\n\n"},
    {"tfe_grad_clip", (PyCFunction)(void (*)(void))grad_clip, FAST,
     "tfe_grad_clip($module, tensors, n, max_norm, norm, stream=None)\n--\n\n"},
    {"tfe_grad_norm_clip", (PyCFunction)(void (*)(void))grad_norm_clip, FAST,
     "tfe_grad_norm_clip($module, tensors, n, max_norm, norm, workspace, workspace_bytes, "
     "stream=None)\n--\n\n"},
    {"tfe_integer_linear", (PyCFunction)(void (*)(void))integer_linear, FAST,
     "tfe_integer_linear($module, x, dtype, ldx, w, w_scales, rows, out_dim, dim, out, "
     "out_dtype, ldo, workspace, workspace_bytes, stream=None)\n--\n\n"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls(void) {
  g_data_ptr = PyUnicode_InternFromString("data_ptr");
  g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
  if (!g_data_ptr || !g_cuda_stream) return nullptr;
  return PyModule_Create(&g_module);
}
