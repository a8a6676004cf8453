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

#define ACCEPT_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ACCEPT_METHOD(compress), ACCEPT_METHOD(decompress), ACCEPT_METHOD(layer_norm), ACCEPT_METHOD(layer_norm_quantize),
    ACCEPT_METHOD(layer_norm_backward), ACCEPT_METHOD(block_quantize), ACCEPT_METHOD(block_matmul),
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
