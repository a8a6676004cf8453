// The device-side calls of the Python binding, for plain tensors: the same checks, pointers and stream as
// binding.py, without the interpreter.  A call with anything out of the ordinary (a tensor subclass, a wrong
// type or size, a tensor without storage) returns kNotHere before anything was done: binding.py then takes it,
// and says what is wrong.
//
// A small tensor's call is host time, nearly all of it the launches, about 3 us each: compressing in one kernel 3.2 us where the host
// is fast, of which 0.1 are the wrapper's in binding.py, and 5.1 where it is slow, in two there 7.7.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>

#include "accept.h"
#include "accept_attention.h"
#include "accept_stage.h"

namespace {

constexpr long kNotHere = -1;
PyObject* g_get_device = nullptr;  // torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
PyObject* g_get_stream = nullptr;

// A descriptor inside the binding's ctypes structure, for the length of a call.
template <typename Desc>
struct View {
  Py_buffer view{};
  bool held = false;
  const Desc* get(PyObject* o) {
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) {
      PyErr_Clear();
      return nullptr;
    }
    held = true;
    return view.len == Py_ssize_t(sizeof(Desc)) ? static_cast<const Desc*>(view.buf) : nullptr;
  }
  ~View() {
    if (held) PyBuffer_Release(&view);
  }
};
using DescView = View<accept_desc>;

bool current_stream(void** stream, long* index = nullptr) {
  PyObject* device = PyObject_CallNoArgs(g_get_device);
  if (device && index) *index = PyLong_AsLong(device);
  PyObject* raw = device ? PyObject_CallOneArg(g_get_stream, device) : nullptr;
  Py_XDECREF(device);
  if (raw) *stream = PyLong_AsVoidPtr(raw);
  Py_XDECREF(raw);
  if (!PyErr_Occurred()) return true;
  PyErr_Clear();
  return false;
}

const at::Tensor* plain_tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

bool fits(const at::Tensor* t, size_t bytes) {
  return t && t->is_cuda() && size_t(t->numel()) * t->element_size() >= bytes && t->is_contiguous();
}
bool fits(const at::Tensor* t, int dtype, int64_t elems) {
  return t && t->scalar_type() == (dtype == ACCEPT_BF16 ? at::kBFloat16 : at::kFloat) && t->is_cuda() &&
         t->numel() >= elems && t->is_contiguous();
}

// compress(desc, x, alpha_prev or None, header, payload, workspace, first) -> status or kNotHere
PyObject* compress(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 7) return PyLong_FromLong(kNotHere);
  try {
    DescView dv;
    const accept_desc* d = dv.get(args[0]);
    size_t hb = 0, pb = 0, wb = 0;
    if (!d || accept_packed_size(d, &hb, &pb) != ACCEPT_OK || accept_workspace_size(d, &wb) != ACCEPT_OK)
      return PyLong_FromLong(kNotHere);
    const bool first = args[6] == Py_True;
    const bool alpha_used = d->scheme == ACCEPT_MBQ && !first;
    const at::Tensor *x = plain_tensor(args[1]), *alpha = args[2] == Py_None ? nullptr : plain_tensor(args[2]);
    const at::Tensor *header = plain_tensor(args[3]), *payload = plain_tensor(args[4]), *ws = plain_tensor(args[5]);
    void* stream = nullptr;
    if (!fits(x, d->in_dtype, d->n * d->m) || !fits(header, hb) || !fits(payload, pb) || !fits(ws, wb) ||
        (alpha_used && !fits(alpha, ACCEPT_F32, d->bits)) || (!alpha && args[2] != Py_None) || !current_stream(&stream))
      return PyLong_FromLong(kNotHere);
    const void* xp = x->data_ptr();
    const float* ap = alpha ? static_cast<const float*>(alpha->data_ptr()) : nullptr;
    void *hp = header->data_ptr(), *pp = payload->data_ptr(), *wp = ws->data_ptr();
    accept_status st;
    Py_BEGIN_ALLOW_THREADS
    st = first ? accept_mbq_compress_first(d, xp, hp, pp, wp, stream) : accept_compress(d, xp, ap, hp, pp, wp, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
  } catch (const std::exception&) {  // a tensor that has no storage, for one
    return PyLong_FromLong(kNotHere);
  }
}

// Other Python threads run on while this lives.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// decompress(desc, header, payload, out or None) -> status, or where there was no `out` the tensor made for it, or kNotHere
PyObject* decompress(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  if (nargs != 4) return PyLong_FromLong(kNotHere);
  try {
    DescView dv;
    const accept_desc* d = dv.get(args[0]);
    size_t hb = 0, pb = 0;
    if (!d || accept_packed_size(d, &hb, &pb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    const at::Tensor *header = plain_tensor(args[1]), *payload = plain_tensor(args[2]);
    const bool make = args[3] == Py_None;
    const at::Tensor* out = make ? nullptr : plain_tensor(args[3]);
    void* stream = nullptr;
    if (!fits(header, hb) || !fits(payload, pb) || (!make && !fits(out, d->out_dtype, d->n * d->m)) || !current_stream(&stream))
      return PyLong_FromLong(kNotHere);
    at::Tensor made;
    if (make) {
      const Unlocked unlocked;  // as in torch.empty: memory that has to be made or freed first waits for the device, and with it for what other threads do for it
      made = at::empty({d->n * d->m}, payload->options().dtype(d->out_dtype == ACCEPT_BF16 ? at::kBFloat16 : at::kFloat));
      out = &made;
    }
    const void *hp = header->data_ptr(), *pp = payload->data_ptr();
    void* op = out->data_ptr();
    accept_status st;
    Py_BEGIN_ALLOW_THREADS
    st = accept_decompress(d, hp, pp, op, stream);
    Py_END_ALLOW_THREADS
    return make && st == ACCEPT_OK ? THPVariable_Wrap(made) : PyLong_FromLong(st);
  } catch (const std::exception&) {
    return PyLong_FromLong(kNotHere);
  }
}

// ---- the stage operators (accept_stage.h): outputs that are not given are made here --------------------------------
constexpr at::ScalarType kScaleType = at::kFloat8_e8m0fnu;
at::ScalarType value_type(int dtype) { return dtype == ACCEPT_BF16 ? at::kBFloat16 : at::kFloat; }
at::ScalarType code_type(int code) { return code == ACCEPT_E5M2 ? at::kFloat8_e5m2 : at::kFloat8_e4m3fn; }
int64_t blocks_of(int64_t length, int64_t by) { return (length + by - 1) / by; }

// What a call's tensors are checked against; `ok` falls and stays where one is not what the descriptor says.
struct Checked {
  long device = -1;
  void* stream = nullptr;
  bool ok = true;

  Checked() { ok = current_stream(&stream, &device); }
  const at::Tensor* get(PyObject* o, bool may_miss) {
    if (o == Py_None) {
      ok = ok && may_miss;
      return nullptr;
    }
    const at::Tensor* t = plain_tensor(o);
    ok = ok && t;
    return t;
  }
  bool here(const at::Tensor* t, at::ScalarType type) {
    return ok = ok && t && t->scalar_type() == type && t->is_cuda() && t->get_device() == device;
  }
  void matrix(const at::Tensor* t, at::ScalarType type, int64_t rows, int64_t cols, int64_t stride) {
    if (!here(t, type)) return;
    if (stride == 0) stride = cols;
    if (t->dim() == 2 && t->size(0) == rows && t->size(1) == cols)
      ok = (rows <= 1 || cols == 0 || t->stride(0) == stride) && (cols <= 1 || rows == 0 || t->stride(1) == 1);
    else
      ok = t->numel() == rows * cols && stride == cols && t->is_contiguous();
  }
  void flat(const at::Tensor* t, at::ScalarType type, int64_t elems) {
    if (here(t, type)) ok = t->numel() == elems && t->is_contiguous();
  }
  // (rows, cols), contiguous: in another order they would be read as another's
  void table(const at::Tensor* t, at::ScalarType type, int64_t rows, int64_t cols) {
    if (here(t, type)) ok = t->dim() == 2 && t->size(0) == rows && t->size(1) == cols && t->is_contiguous();
  }
  // codes whose rows are readable `reach` bytes far
  void codes(const at::Tensor* t, int code, int64_t rows, int64_t cols, int64_t stride, int64_t reach) {
    if (!here(t, code_type(code))) return;
    ok = t->dim() == 2 && t->size(0) == rows && t->size(1) == cols;
    if (!ok || rows == 0 || cols == 0) return;
    ok = (rows <= 1 || t->stride(0) == stride) && (cols <= 1 || t->stride(1) == 1) &&
         reinterpret_cast<uintptr_t>(t->data_ptr()) % 16 == 0 &&
         t->storage_offset() + (rows - 1) * stride + reach <= int64_t(t->storage().nbytes());
  }
};

at::Tensor make(const at::Tensor& like, at::IntArrayRef size, at::ScalarType type) {
  const Unlocked unlocked;
  return at::empty(size, like.options().dtype(type));
}
at::Tensor make_rows(const at::Tensor& like, int64_t rows, int64_t cols, int64_t stride, at::ScalarType type) {
  at::Tensor t = make(like, {rows, stride}, type);
  return stride == cols ? t : t.narrow(1, 0, cols);
}
at::Tensor make_matrix(const at::Tensor& x, int64_t rows, int64_t cols, int64_t stride, at::ScalarType type) {
  return stride == 0 || stride == cols ? make(x, x.sizes(), type) : make_rows(x, rows, cols, stride, type);
}
void* pointer(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }

PyObject* tuple_of(std::initializer_list<const at::Tensor*> tensors) {
  PyObject* r = PyTuple_New(Py_ssize_t(tensors.size()));
  Py_ssize_t i = 0;
  for (const at::Tensor* t : tensors) {
    PyObject* o = t ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
    if (!r || !o) {
      Py_XDECREF(o);
      Py_XDECREF(r);
      return nullptr;
    }
    PyTuple_SET_ITEM(r, i++, o);
  }
  return r;
}

// A call into the library, other Python threads running on.
template <typename F>
accept_status call(const F& f) {
  const Unlocked unlocked;
  return f();
}

template <typename F>
PyObject* guarded(const F& f) {
  try {
    return f();
  } catch (const std::exception&) {  // a tensor that has no storage, no memory for an output: the slow way says what it is
    return PyLong_FromLong(kNotHere);
  }
}

// layer_norm(desc, x, weight, bias, y, stats) -> (y, stats), a status or kNotHere
PyObject* layer_norm(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_norm_desc> dv;
    const accept_norm_desc* d = nargs == 6 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!d || accept_norm_workspace_size(d, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    Checked c;
    const at::Tensor *x = c.get(args[1], false), *w = c.get(args[2], true), *b = c.get(args[3], true), *y = c.get(args[4], true),
                     *stats = c.get(args[5], true);
    const at::ScalarType param = value_type(d->param_dtype), out = value_type(d->y_dtype);
    c.matrix(x, value_type(d->x_dtype), d->rows, d->cols, d->x_stride);
    if (w) c.flat(w, param, d->cols);
    if (b) c.flat(b, param, d->cols);
    if (y) c.matrix(y, out, d->rows, d->cols, d->y_stride);
    if (stats) c.table(stats, at::kFloat, 2, d->rows);
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor my, ms;
    if (!y) my = make_matrix(*x, d->rows, d->cols, d->y_stride, out), y = &my;
    if (!stats) ms = make(*x, {2, d->rows}, at::kFloat), stats = &ms;
    void *xp = pointer(x), *wp = pointer(w), *bp = pointer(b), *yp = pointer(y), *sp = pointer(stats);
    const accept_status st = call([&] { return accept_layer_norm(d, xp, wp, bp, yp, static_cast<float*>(sp), c.stream); });
    return st == ACCEPT_OK ? tuple_of({y, stats}) : PyLong_FromLong(st);
  });
}

// layer_norm_quantize(desc, x, weight, bias, codes, scales, stats) -> (codes, scales, stats), a status or kNotHere
PyObject* layer_norm_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_norm_desc> dv;
    const accept_norm_desc* d = nargs == 7 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!d || accept_norm_workspace_size(d, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    Checked c;
    const at::Tensor *x = c.get(args[1], false), *w = c.get(args[2], true), *b = c.get(args[3], true), *codes = c.get(args[4], true),
                     *scales = c.get(args[5], true), *stats = c.get(args[6], true);
    const at::ScalarType param = value_type(d->param_dtype);
    const int64_t stride = accept_block_stride(d->cols), blocks = blocks_of(d->cols, 128);
    c.matrix(x, value_type(d->x_dtype), d->rows, d->cols, d->x_stride);
    if (w) c.flat(w, param, d->cols);
    if (b) c.flat(b, param, d->cols);
    if (codes) c.codes(codes, d->code, d->rows, d->cols, stride, stride);
    if (scales) c.table(scales, kScaleType, blocks, d->rows);
    if (stats) c.table(stats, at::kFloat, 2, d->rows);
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor mc, me, ms;
    if (!codes) mc = make_rows(*x, d->rows, d->cols, stride, code_type(d->code)), codes = &mc;
    if (!scales) me = make(*x, {blocks, d->rows}, kScaleType), scales = &me;
    if (!stats) ms = make(*x, {2, d->rows}, at::kFloat), stats = &ms;
    void *xp = pointer(x), *wp = pointer(w), *bp = pointer(b), *cp = pointer(codes), *ep = pointer(scales), *sp = pointer(stats);
    const accept_status st =
        call([&] { return accept_layer_norm_quantize(d, xp, wp, bp, cp, ep, static_cast<float*>(sp), c.stream); });
    return st == ACCEPT_OK ? tuple_of({codes, scales, stats}) : PyLong_FromLong(st);
  });
}

// layer_norm_backward(desc, dy, x, weight, stats, dx, dweight, dbias, need_weight, need_bias, workspace) -> (dx, dweight, dbias), a status
// or kNotHere
PyObject* layer_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_norm_desc> dv;
    const accept_norm_desc* d = nargs == 11 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!d || accept_norm_workspace_size(d, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    if (!PyBool_Check(args[8]) || !PyBool_Check(args[9])) return PyLong_FromLong(kNotHere);
    const bool need_weight = args[8] == Py_True, need_bias = args[9] == Py_True;
    Checked c;
    const at::Tensor *dy = c.get(args[1], false), *x = c.get(args[2], false), *w = c.get(args[3], true), *stats = c.get(args[4], false),
                     *dx = c.get(args[5], true), *dw = c.get(args[6], true), *db = c.get(args[7], true), *ws = c.get(args[10], true);
    const at::ScalarType type = value_type(d->x_dtype), param = value_type(d->param_dtype);
    c.matrix(dy, value_type(d->y_dtype), d->rows, d->cols, d->y_stride);
    c.matrix(x, type, d->rows, d->cols, d->x_stride);
    if (w) c.flat(w, param, d->cols);
    c.table(stats, at::kFloat, 2, d->rows);
    if (dx) c.matrix(dx, type, d->rows, d->cols, d->dx_stride);
    if (!need_weight) dw = nullptr;
    if (!need_bias) db = nullptr;
    if (dw) c.flat(dw, param, d->cols);
    if (db) c.flat(db, param, d->cols);
    const bool sums = need_weight || need_bias;
    if (sums && ws) c.ok = c.ok && fits(ws, wb) && ws->get_device() == c.device;
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor mx, mw, mb, mws;
    if (!dx) mx = make_matrix(*x, d->rows, d->cols, d->dx_stride, type), dx = &mx;
    if (need_weight && !dw) mw = make(*x, {d->cols}, param), dw = &mw;
    if (need_bias && !db) mb = make(*x, {d->cols}, param), db = &mb;
    if (sums && !ws) mws = make(*x, {int64_t(wb)}, at::kByte), ws = &mws;
    void *yp = pointer(dy), *xp = pointer(x), *wp = pointer(w), *sp = pointer(stats), *dp = pointer(dx), *dwp = pointer(dw),
         *dbp = pointer(db), *wsp = sums ? pointer(ws) : nullptr;
    const accept_status st = call([&] {
      return accept_layer_norm_backward(d, yp, xp, wp, static_cast<const float*>(sp), dp, dwp, dbp, wsp, c.stream);
    });
    return st == ACCEPT_OK ? tuple_of({dx, dw, db}) : PyLong_FromLong(st);
  });
}

// block_quantize(desc, x, rowwise, colwise, codes, scales, codes_t, scales_t) -> the last four, a status or kNotHere
PyObject* block_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_block_desc> dv;
    const accept_block_desc* d = nargs == 8 ? dv.get(args[0]) : nullptr;
    if (!d || !PyBool_Check(args[2]) || !PyBool_Check(args[3])) return PyLong_FromLong(kNotHere);
    const bool rowwise = args[2] == Py_True, colwise = args[3] == Py_True;
    if (d->rows <= 0 || d->cols <= 0 || d->rows > INT32_MAX || d->cols > INT32_MAX || (d->group != 1 && d->group != 128) ||
        (!rowwise && !colwise))
      return PyLong_FromLong(kNotHere);
    Checked c;
    const at::Tensor *x = c.get(args[1], false), *given[4], **g = given;
    for (int i = 0; i < 4; ++i) given[i] = (i < 2 ? rowwise : colwise) ? c.get(args[4 + i], true) : nullptr;
    const int64_t rows = d->rows, cols = d->cols, stride = accept_block_stride(cols), stride_t = accept_block_stride(rows);
    const int64_t eb = blocks_of(cols, 128), er = blocks_of(rows, d->group), tb = blocks_of(rows, 128), tr = blocks_of(cols, d->group);
    c.matrix(x, value_type(d->in_dtype), rows, cols, d->x_stride);
    if (g[0]) c.codes(g[0], d->code, rows, cols, stride, stride);
    if (g[1]) c.table(g[1], kScaleType, eb, er);
    if (g[2]) c.codes(g[2], d->code, cols, rows, stride_t, stride_t);
    if (g[3]) c.table(g[3], kScaleType, tb, tr);
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor made[4];
    if (rowwise && !g[0]) made[0] = make_rows(*x, rows, cols, stride, code_type(d->code)), g[0] = &made[0];
    if (rowwise && !g[1]) made[1] = make(*x, {eb, er}, kScaleType), g[1] = &made[1];
    if (colwise && !g[2]) made[2] = make_rows(*x, cols, rows, stride_t, code_type(d->code)), g[2] = &made[2];
    if (colwise && !g[3]) made[3] = make(*x, {tb, tr}, kScaleType), g[3] = &made[3];
    void *xp = pointer(x), *p0 = pointer(g[0]), *p1 = pointer(g[1]), *p2 = pointer(g[2]), *p3 = pointer(g[3]);
    const accept_status st = call([&] { return accept_block_quantize(d, xp, p0, p1, p2, p3, c.stream); });
    return st == ACCEPT_OK ? tuple_of({g[0], g[1], g[2], g[3]}) : PyLong_FromLong(st);
  });
}

// block_matmul(desc, a, a_scales, b, b_scales, y, workspace) -> (y,), a status or kNotHere
PyObject* block_matmul(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_matmul_desc> dv;
    const accept_matmul_desc* d = nargs == 7 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!d || accept_matmul_workspace_size(d, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    Checked c;
    const at::Tensor *a = c.get(args[1], false), *sa = c.get(args[2], false), *b = c.get(args[3], false), *sb = c.get(args[4], false),
                     *y = c.get(args[5], true), *ws = c.get(args[6], true);
    const int64_t whole = accept_block_stride(d->k), reach = blocks_of(d->k, 16) * 16, blocks = blocks_of(d->k, 128);
    const at::ScalarType out = value_type(d->out_dtype);
    c.codes(a, d->a_code, d->m, d->k, d->a_stride ? d->a_stride : whole, reach);
    c.codes(b, d->b_code, d->n, d->k, d->b_stride ? d->b_stride : whole, reach);
    c.table(sa, kScaleType, blocks, blocks_of(d->m, d->a_group));
    c.table(sb, kScaleType, blocks, blocks_of(d->n, d->b_group));
    if (y) c.matrix(y, out, d->m, d->n, d->y_stride);
    if (wb && ws) c.ok = c.ok && fits(ws, wb) && ws->get_device() == c.device;
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor my, mws;
    if (!y) my = make_rows(*a, d->m, d->n, d->y_stride ? d->y_stride : d->n, out), y = &my;
    if (wb && !ws) mws = make(*a, {int64_t(wb)}, at::kByte), ws = &mws;
    void *ap = pointer(a), *sap = pointer(sa), *bp = pointer(b), *sbp = pointer(sb), *yp = pointer(y), *wsp = wb ? pointer(ws) : nullptr;
    const accept_status st = call([&] { return accept_block_matmul(d, ap, sap, bp, sbp, yp, wsp, c.stream); });
    return st == ACCEPT_OK ? tuple_of({y}) : PyLong_FromLong(st);
  });
}

// ---- the attention operators (accept_attention.h) ---------------------------------------------------------------------
// What a call allocates holds zeros for tokens of no sequence; what it is given follows the descriptor.
struct Tokens {
  Checked& c;
  at::ScalarType type;
  // (tokens, heads, head) or (tokens, heads * head), tokens `stride` (0: as many) apart, 16-byte aligned
  void operator()(const at::Tensor* t, int64_t tokens, int64_t heads, int64_t head, int64_t stride) const {
    if (!c.here(t, type)) return;
    const int64_t whole = heads * head;
    const bool three = t->dim() == 3;
    if (!three && t->dim() != 2) {
      c.ok = false;
      return;
    }
    c.ok = t->size(0) == tokens && (three ? t->size(1) == heads && t->size(2) == head : t->size(1) == whole);
    if (!c.ok || tokens == 0) return;
    c.ok = t->stride(-1) == 1 && (!three || heads == 1 || t->stride(1) == head) && (tokens == 1 || t->stride(0) == (stride ? stride : whole)) &&
           reinterpret_cast<uintptr_t>(t->data_ptr()) % 16 == 0;
  }
};
void ints(Checked& c, const at::Tensor* t, int64_t size) { c.flat(t, at::kInt, size); }
bool shared_out(const at::Tensor* offsets, int64_t sequences, int64_t tokens) {
  return offsets || (sequences > 0 ? tokens % sequences == 0 : tokens == 0);
}
at::Tensor make_tokens(const at::Tensor& like, int64_t tokens, int64_t heads, int64_t head, int64_t stride, at::ScalarType type) {
  const int64_t whole = heads * head;
  if (stride == 0 || stride == whole) return make(like, {tokens, heads, head}, type);
  return make(like, {tokens, stride}, type).narrow(1, 0, whole).unflatten(1, {heads, head});
}
const int32_t* int_pointer(const at::Tensor* t) { return t ? static_cast<const int32_t*>(t->data_ptr()) : nullptr; }

// rotate(desc, x, frequencies, offsets, positions, y) -> (y,), a status or kNotHere
PyObject* rotate(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_rotate_desc> dv;
    const accept_rotate_desc* given = nargs == 6 ? dv.get(args[0]) : nullptr;
    if (!given || (given->dtype != ACCEPT_F32 && given->dtype != ACCEPT_BF16) || given->sequences < 0 || given->tokens < 0 || given->heads < 1 ||
        given->head_size < 1 || given->y_stride < 0)
      return PyLong_FromLong(kNotHere);
    accept_rotate_desc d = *given;
    Checked c;
    const at::Tensor *x = c.get(args[1], false), *f = c.get(args[2], d.rotated == 0), *off = c.get(args[3], true), *pos = c.get(args[4], true),
                     *y = c.get(args[5], true);
    const Tokens tokens{c, value_type(d.dtype)};
    tokens(x, d.tokens, d.heads, d.head_size, d.x_stride);
    if (f) c.flat(f, at::kFloat, d.rotated / 2);
    if (off) ints(c, off, d.sequences + 1);
    if (pos) ints(c, pos, d.tokens);
    if (!pos) c.ok = c.ok && shared_out(off, d.sequences, d.tokens);
    if (y) tokens(y, d.tokens, d.heads, d.head_size, d.y_stride);
    if (!c.ok || (d.y_stride && d.y_stride < int64_t(d.heads) * d.head_size)) return PyLong_FromLong(kNotHere);
    at::Tensor my;
    if (!y) {
      my = make_tokens(*x, d.tokens, d.heads, d.head_size, d.y_stride, x->scalar_type()), y = &my;
      if (off) d.rest = ACCEPT_REST_ZEROS;
    }
    void *xp = pointer(x), *fp = pointer(f), *yp = pointer(y);
    const int32_t *op = int_pointer(off), *pp = int_pointer(pos);
    const accept_status st = call([&] { return accept_rotate(&d, xp, static_cast<const float*>(fp), op, pp, yp, c.stream); });
    return st == ACCEPT_OK ? tuple_of({y}) : PyLong_FromLong(st);
  });
}

// attention(desc, q, k, v, q_offsets, k_offsets, o, lse, workspace) -> (o, lse), a status or kNotHere
PyObject* attention(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_attention_desc> dv;
    const accept_attention_desc* given = nargs == 9 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!given || accept_attention_workspace_size(given, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    accept_attention_desc d = *given;
    Checked c;
    const at::Tensor *q = c.get(args[1], false), *k = c.get(args[2], false), *v = c.get(args[3], false), *qo = c.get(args[4], true),
                     *ko = c.get(args[5], true), *o = c.get(args[6], true), *lse = c.get(args[7], true), *ws = c.get(args[8], true);
    const Tokens tokens{c, value_type(d.dtype)};
    tokens(q, d.q_tokens, d.heads, d.head_size, d.q_stride);
    tokens(k, d.k_tokens, d.kv_heads, d.head_size, d.k_stride);
    tokens(v, d.k_tokens, d.kv_heads, d.head_size, d.v_stride);
    if (qo) ints(c, qo, d.sequences + 1);
    if (ko) ints(c, ko, d.sequences + 1);
    c.ok = c.ok && shared_out(qo, d.sequences, d.q_tokens) && shared_out(ko, d.sequences, d.k_tokens);
    if (o) tokens(o, d.q_tokens, d.heads, d.head_size, d.o_stride);
    if (lse) c.table(lse, at::kFloat, d.heads, d.q_tokens);
    if (wb && ws) c.ok = c.ok && fits(ws, wb) && ws->get_device() == c.device;
    // one of the two made here and the other given: the slow way's, as their rests differ
    if (!c.ok || (qo && !o != !lse)) return PyLong_FromLong(kNotHere);
    at::Tensor mo, ml, mws;
    if (!o) {
      mo = make_tokens(*q, d.q_tokens, d.heads, d.head_size, d.o_stride, q->scalar_type()), o = &mo;
      if (qo) d.rest = ACCEPT_REST_ZEROS;
    }
    if (!lse) ml = make(*q, {d.heads, d.q_tokens}, at::kFloat), lse = &ml;
    if (wb && !ws) mws = make(*q, {int64_t(wb)}, at::kByte), ws = &mws;
    void *qp = pointer(q), *kp = pointer(k), *vp = pointer(v), *op = pointer(o), *lp = pointer(lse), *wp = wb ? pointer(ws) : nullptr;
    const int32_t *qop = int_pointer(qo), *kop = int_pointer(ko);
    const accept_status st =
        call([&] { return accept_attention(&d, qp, kp, vp, qop, kop, op, static_cast<float*>(lp), wp, c.stream); });
    return st == ACCEPT_OK ? tuple_of({o, lse}) : PyLong_FromLong(st);
  });
}

// attention_backward(desc, do, q, k, v, o, lse, q_offsets, k_offsets, dq, dk, dv, workspace) -> (dq, dk, dv), a status or kNotHere
PyObject* attention_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_attention_desc> dv;
    const accept_attention_desc* given = nargs == 13 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!given || accept_attention_backward_workspace_size(given, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    accept_attention_desc d = *given;
    // all three gradients made here, or all given: the slow way takes what lies between
    const int missing = (args[9] == Py_None) + (args[10] == Py_None) + (args[11] == Py_None);
    if (missing != 0 && missing != 3) return PyLong_FromLong(kNotHere);
    Checked c;
    const at::Tensor *dout = c.get(args[1], false), *q = c.get(args[2], false), *k = c.get(args[3], false), *v = c.get(args[4], false),
                     *o = c.get(args[5], false), *lse = c.get(args[6], false), *qo = c.get(args[7], true), *ko = c.get(args[8], true),
                     *dq = c.get(args[9], true), *dk = c.get(args[10], true), *dvt = c.get(args[11], true), *ws = c.get(args[12], true);
    const Tokens tokens{c, value_type(d.dtype)};
    tokens(q, d.q_tokens, d.heads, d.head_size, d.q_stride);
    tokens(k, d.k_tokens, d.kv_heads, d.head_size, d.k_stride);
    tokens(v, d.k_tokens, d.kv_heads, d.head_size, d.v_stride);
    tokens(o, d.q_tokens, d.heads, d.head_size, d.o_stride);
    tokens(dout, d.q_tokens, d.heads, d.head_size, d.o_stride);
    c.table(lse, at::kFloat, d.heads, d.q_tokens);
    if (qo) ints(c, qo, d.sequences + 1);
    if (ko) ints(c, ko, d.sequences + 1);
    c.ok = c.ok && shared_out(qo, d.sequences, d.q_tokens) && shared_out(ko, d.sequences, d.k_tokens);
    if (!missing) {
      tokens(dq, d.q_tokens, d.heads, d.head_size, d.dq_stride);
      tokens(dk, d.k_tokens, d.kv_heads, d.head_size, d.dk_stride);
      tokens(dvt, d.k_tokens, d.kv_heads, d.head_size, d.dv_stride);
    }
    if (wb && ws) c.ok = c.ok && fits(ws, wb) && ws->get_device() == c.device;
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor mq, mk, mv, mws;
    if (missing) {
      mq = make_tokens(*q, d.q_tokens, d.heads, d.head_size, d.dq_stride, q->scalar_type()), dq = &mq;
      mk = make_tokens(*q, d.k_tokens, d.kv_heads, d.head_size, d.dk_stride, q->scalar_type()), dk = &mk;
      mv = make_tokens(*q, d.k_tokens, d.kv_heads, d.head_size, d.dv_stride, q->scalar_type()), dvt = &mv;
      if (qo || ko) d.rest = ACCEPT_REST_ZEROS;
    }
    if (wb && !ws) mws = make(*q, {int64_t(wb)}, at::kByte), ws = &mws;
    void *dp = pointer(dout), *qp = pointer(q), *kp = pointer(k), *vp = pointer(v), *op = pointer(o), *lp = pointer(lse), *dqp = pointer(dq),
         *dkp = pointer(dk), *dvp = pointer(dvt), *wp = wb ? pointer(ws) : nullptr;
    const int32_t *qop = int_pointer(qo), *kop = int_pointer(ko);
    const accept_status st = call([&] {
      return accept_attention_backward(&d, dp, qp, kp, vp, op, static_cast<const float*>(lp), qop, kop, dqp, dkp, dvp, wp, c.stream);
    });
    return st == ACCEPT_OK ? tuple_of({dq, dk, dvt}) : PyLong_FromLong(st);
  });
}

// The caches, table, lengths and offsets of a call.
void check_cache(Checked& c, const accept_cache_desc& d, const at::Tensor* k_cache, const at::Tensor* v_cache, const at::Tensor* table,
                 const at::Tensor* lengths, const at::Tensor* offsets) {
  for (const at::Tensor* t : {k_cache, v_cache})
    if (c.here(t, value_type(d.dtype)))
      c.ok = t->dim() == 4 && t->size(0) == d.pages && t->size(1) == d.kv_heads && t->size(2) == d.page_size && t->size(3) == d.head_size &&
             t->is_contiguous() && reinterpret_cast<uintptr_t>(t->data_ptr()) % 16 == 0;
  c.table(table, at::kInt, d.sequences, d.table_pages);
  ints(c, lengths, d.sequences);
  if (offsets) ints(c, offsets, d.sequences + 1);
  c.ok = c.ok && shared_out(offsets, d.sequences, d.tokens);
}

// cache_append(desc, q, k, v, k_cache, v_cache, table, lengths, offsets, positions, frequencies, q_out) -> (q_out or None,), a status or kNotHere
PyObject* cache_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_cache_desc> dv;
    const accept_cache_desc* given = nargs == 12 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!given || accept_cache_workspace_size(given, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    accept_cache_desc d = *given;
    Checked c;
    const at::Tensor *q = c.get(args[1], true), *k = c.get(args[2], false), *v = c.get(args[3], false), *kc = c.get(args[4], false),
                     *vc = c.get(args[5], false), *table = c.get(args[6], false), *lengths = c.get(args[7], false), *off = c.get(args[8], true),
                     *pos = c.get(args[9], true), *f = c.get(args[10], d.rotated == 0), *out = c.get(args[11], true);
    if (!c.ok) return PyLong_FromLong(kNotHere);
    check_cache(c, d, kc, vc, table, lengths, off);
    const Tokens tokens{c, value_type(d.dtype)};
    if (q) tokens(q, d.tokens, d.heads, d.head_size, d.q_stride);
    tokens(k, d.tokens, d.kv_heads, d.head_size, d.k_stride);
    tokens(v, d.tokens, d.kv_heads, d.head_size, d.v_stride);
    if (pos) ints(c, pos, d.tokens);
    if (f) c.flat(f, at::kFloat, d.rotated / 2);
    if (out) tokens(out, d.tokens, d.heads, d.head_size, d.qo_stride);
    if (!c.ok || (out && !q)) return PyLong_FromLong(kNotHere);
    at::Tensor mo;
    if (q && !out) {
      mo = make_tokens(*q, d.tokens, d.heads, d.head_size, d.qo_stride, q->scalar_type()), out = &mo;
      if (off) d.rest = ACCEPT_REST_ZEROS;
    }
    void *qp = pointer(q), *kp = pointer(k), *vp = pointer(v), *fp = pointer(f), *op = pointer(out), *kcp = pointer(kc), *vcp = pointer(vc);
    const int32_t *offp = int_pointer(off), *lp = int_pointer(lengths), *pp = int_pointer(pos), *tp = int_pointer(table);
    const accept_status st =
        call([&] { return accept_cache_append(&d, qp, kp, vp, static_cast<const float*>(fp), offp, lp, pp, tp, op, kcp, vcp, c.stream); });
    return st == ACCEPT_OK ? tuple_of({out}) : PyLong_FromLong(st);
  });
}

// cache_attention(desc, q, k_cache, v_cache, table, lengths, offsets, tree, o, workspace) -> (o,), a status or kNotHere
PyObject* cache_attention(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  return guarded([&]() -> PyObject* {
    View<accept_cache_desc> dv;
    const accept_cache_desc* given = nargs == 10 ? dv.get(args[0]) : nullptr;
    size_t wb = 0;
    if (!given || accept_cache_workspace_size(given, &wb) != ACCEPT_OK) return PyLong_FromLong(kNotHere);
    accept_cache_desc d = *given;
    Checked c;
    const at::Tensor *q = c.get(args[1], false), *kc = c.get(args[2], false), *vc = c.get(args[3], false), *table = c.get(args[4], false),
                     *lengths = c.get(args[5], false), *off = c.get(args[6], true), *tree = c.get(args[7], d.tree_words == 0),
                     *o = c.get(args[8], true), *ws = c.get(args[9], true);
    if (!c.ok || (tree && d.tree_words == 0)) return PyLong_FromLong(kNotHere);
    check_cache(c, d, kc, vc, table, lengths, off);
    const Tokens tokens{c, value_type(d.dtype)};
    tokens(q, d.tokens, d.heads, d.head_size, d.q_stride);
    if (tree) c.table(tree, at::kLong, d.tokens, d.tree_words);
    if (o) tokens(o, d.tokens, d.heads, d.head_size, d.o_stride);
    if (wb && ws) c.ok = c.ok && fits(ws, wb) && ws->get_device() == c.device;
    if (!c.ok) return PyLong_FromLong(kNotHere);
    at::Tensor mo, mws;
    if (!o) {
      mo = make_tokens(*q, d.tokens, d.heads, d.head_size, d.o_stride, q->scalar_type()), o = &mo;
      if (off) d.rest = ACCEPT_REST_ZEROS;
    }
    if (wb && !ws) mws = make(*q, {int64_t(wb)}, at::kByte), ws = &mws;
    void *qp = pointer(q), *kcp = pointer(kc), *vcp = pointer(vc), *op = pointer(o), *wp = wb ? pointer(ws) : nullptr, *tp = pointer(tree);
    const int32_t *offp = int_pointer(off), *lp = int_pointer(lengths), *tabp = int_pointer(table);
    const accept_status st =
        call([&] { return accept_cache_attention(&d, qp, kcp, vcp, offp, lp, tabp, static_cast<const uint64_t*>(tp), op, wp, c.stream); });
    return st == ACCEPT_OK ? tuple_of({o}) : PyLong_FromLong(st);
  });
}

#define ACCEPT_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ACCEPT_METHOD(compress), ACCEPT_METHOD(decompress), ACCEPT_METHOD(layer_norm), ACCEPT_METHOD(layer_norm_quantize),
    ACCEPT_METHOD(layer_norm_backward), ACCEPT_METHOD(block_quantize), ACCEPT_METHOD(block_matmul),
    ACCEPT_METHOD(rotate), ACCEPT_METHOD(attention), ACCEPT_METHOD(attention_backward), ACCEPT_METHOD(cache_append),
    ACCEPT_METHOD(cache_attention),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
  PyObject* torch_c = PyImport_ImportModule("torch._C");
  if (!torch_c) return nullptr;
  g_get_device = PyObject_GetAttrString(torch_c, "_cuda_getDevice");
  g_get_stream = PyObject_GetAttrString(torch_c, "_cuda_getCurrentRawStream");
  Py_DECREF(torch_c);
  if (!g_get_device || !g_get_stream) return nullptr;
  return PyModule_Create(&module_def);
}
