// Host side of the Python entry points that run once per request: argument checks, descriptor
// tables, output and workspace tensors, and the call into the C-ABI (include/kan.h), without a trip
// through the interpreter for each of them.
//
// What bounds a small call is this path and not the GPU: a launch costs the host 2.0-2.5 us on this
// stack, and the ctypes form of the binding (a descriptor array built in Python, the stream looked up as a
// torch.cuda.Stream object, one ctypes conversion per argument, torch.full for the output) added 5.4 us
// to a call with buffers of its own and 14 us to one without (2 x 17 us for the descriptors of fifty
// heads), where its two launches themselves take 5-6 us.  Host time per call, ctypes form and this one: a
// two-layer head at batch 1 with kept buffers 11.3 and 6.8 us; one 64 x 32 layer with neither workspace nor
// output given 20.0 and 9.0 (its GPU work 7.7); fifty two-layer heads 33.5 and 18.8.
//
// The functions take the objects of the binding (VQLayer, tensors) as they are and return the output,
// or the kan_status as an int when the call was refused.

#include <ATen/ops/empty.h>
#include <ATen/ops/full.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <initializer_list>

#include "../../include/kan.h"

namespace {

PyObject* g_desc_name = nullptr;        // "desc": the attribute that holds a layer's C descriptor
PyObject* g_raw_stream = nullptr;       // torch._C._cuda_getCurrentRawStream

typedef c10::SmallVector<kan_vq_layer, 8> Table;

// Copies the descriptor of one VQLayer; false with a Python error set.
bool read_desc(PyObject* layer, kan_vq_layer* out) {
  PyObject* desc = PyObject_GetAttr(layer, g_desc_name);
  if (!desc) return false;
  Py_buffer view;
  const int got = PyObject_GetBuffer(desc, &view, PyBUF_SIMPLE);
  Py_DECREF(desc);
  if (got != 0) return false;
  const bool fits = view.len == (Py_ssize_t)sizeof(kan_vq_layer);
  if (fits) memcpy(out, view.buf, sizeof(kan_vq_layer));
  PyBuffer_Release(&view);
  if (!fits) PyErr_SetString(PyExc_TypeError, "desc is not a kan_vq_layer");
  return fits;
}

// heads: sequence (heads) of sequences (layers) of VQLayer -> table [n_heads][n_layers].
bool read_heads(PyObject* heads, Table* table, int32_t* n_layers, int32_t* n_heads) {
  PyObject* hs = PySequence_Fast(heads, "heads: a list of heads, each a list of VQLayer");
  if (!hs) return false;
  const Py_ssize_t H = PySequence_Fast_GET_SIZE(hs);
  Py_ssize_t N = 0;
  bool ok = true;
  for (Py_ssize_t h = 0; ok && h < H; ++h) {
    PyObject* ls = PySequence_Fast(PySequence_Fast_GET_ITEM(hs, h), "a head is a list of VQLayer");
    if (!ls) {
      ok = false;
      break;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(ls);
    if (h == 0) {
      N = n;
      table->reserve((size_t)(H * N));
    }
    if (n != N) {
      PyErr_SetString(PyExc_AssertionError, "every head has the same number of layers");
      ok = false;
    }
    for (Py_ssize_t l = 0; ok && l < n; ++l) {
      table->emplace_back();
      ok = read_desc(PySequence_Fast_GET_ITEM(ls, l), &table->back());
    }
    Py_DECREF(ls);
  }
  Py_DECREF(hs);
  if (ok && (H == 0 || N == 0)) {
    PyErr_SetString(PyExc_IndexError, "no heads or no layers");
    ok = false;
  }
  *n_layers = (int32_t)N;
  *n_heads = (int32_t)H;
  return ok;
}

const at::Tensor* tensor_of(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s: a tensor is expected", what);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}

// Like the rest of the binding, calls go to the current stream of the current device.
bool current_stream(void** out) {
  const c10::Device dev = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice();
  PyObject* index = PyLong_FromLong(dev.index());
  PyObject* raw = index ? PyObject_CallFunctionObjArgs(g_raw_stream, index, nullptr) : nullptr;
  Py_XDECREF(index);
  if (!raw) return false;
  *out = PyLong_AsVoidPtr(raw);
  Py_DECREF(raw);
  return !(*out == nullptr && PyErr_Occurred());
}

bool check_floats(const at::Tensor& t, const char* what) {
  if (t.scalar_type() == at::kFloat && t.is_contiguous()) return true;
  PyErr_Format(PyExc_AssertionError, "%s: float32 and contiguous", what);
  return false;
}

// Workspace and output of one call: the caller's tensors, or tensors of its own.
struct Buffers {
  at::Tensor ws_own, y_own;
  void* ws = nullptr;
  size_t ws_bytes = 0;
  void* y = nullptr;
  PyObject* y_obj = nullptr;        // borrowed: the caller's output

  bool use_ws(PyObject* o, size_t need, const at::Tensor& like) {
    if (o != Py_None) {
      const at::Tensor* t = tensor_of(o, "ws");
      if (!t) return false;
      ws = t->data_ptr();
      ws_bytes = (size_t)t->numel();
    } else if (need > 0) {
      ws_own = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
      ws = ws_own.data_ptr();
      ws_bytes = need;
    }
    return true;
  }
  bool use_y(PyObject* o, at::IntArrayRef shape, const at::Tensor& like) {
    if (o != Py_None) {
      const at::Tensor* t = tensor_of(o, "y");
      if (!t) return false;
      y = t->data_ptr();
      y_obj = o;
    } else {
      y_own = at::empty(shape, like.options());
      y = y_own.data_ptr();
    }
    return true;
  }
  PyObject* result(kan_status st) {
    if (st != KAN_OK) return PyLong_FromLong(st);
    if (y_obj) {
      Py_INCREF(y_obj);
      return y_obj;
    }
    return THPVariable_Wrap(std::move(y_own));
  }
};

PyObject* forward(const Table& table, int32_t n_layers, int32_t n_heads, const at::Tensor& x, long path, PyObject* ws,
                  PyObject* y, bool is_static, bool one_layer) {
  const int64_t B = x.size(0);
  Buffers b;
  if (!is_static) {
    size_t need = 0;
    if (ws == Py_None) {
      need = kan_vq_workspace_bytes(table.data(), n_layers, n_heads, B, (int32_t)path);
      if (need == (size_t)-1) need = 0;        // the forward call reports the precise status
    }
    if (!b.use_ws(ws, need, x)) return nullptr;
  }
  const int64_t out = table[n_layers - 1].out;
  if (!(one_layer ? b.use_y(y, {B, out}, x) : b.use_y(y, {n_heads, B, out}, x))) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const float* xp = (const float*)x.data_ptr();
  kan_status st;
  Py_BEGIN_ALLOW_THREADS
  st = is_static ? kan_vq_head_forward_static(table.data(), n_layers, n_heads, xp, B, (float*)b.y, (int32_t)path, stream)
                 : kan_vq_head_forward(table.data(), n_layers, n_heads, xp, B, (float*)b.y, b.ws, b.ws_bytes, (int32_t)path,
                                       stream);
  Py_END_ALLOW_THREADS
  return b.result(st);
}

bool arity(Py_ssize_t n, Py_ssize_t want) {
  if (n == want) return true;
  PyErr_Format(PyExc_TypeError, "%zd arguments, got %zd", want, n);
  return false;
}

// layer_forward(layer, x, path, ws, y)
PyObject* layer_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 5)) return nullptr;
  const at::Tensor* x = tensor_of(a[1], "x");
  if (!x || !check_floats(*x, "x")) return nullptr;
  Table table(1);
  if (!read_desc(a[0], &table[0])) return nullptr;
  if (x->dim() != 2 || x->size(1) != table[0].in) {
    PyErr_SetString(PyExc_AssertionError, "x: [batch][inputs of the layer]");
    return nullptr;
  }
  const long path = PyLong_AsLong(a[2]);
  if (path == -1 && PyErr_Occurred()) return nullptr;
  return forward(table, 1, 1, *x, path, a[3], a[4], false, true);
  END_HANDLE_TH_ERRORS
}

PyObject* heads_call(PyObject* heads, PyObject* xo, PyObject* patho, PyObject* ws, PyObject* y, bool is_static) {
  const at::Tensor* x = tensor_of(xo, "x");
  if (!x || !check_floats(*x, "x")) return nullptr;
  if (x->dim() < 1) {
    PyErr_SetString(PyExc_IndexError, "x: [batch][inputs]");
    return nullptr;
  }
  Table table;
  int32_t n_layers, n_heads;
  if (!read_heads(heads, &table, &n_layers, &n_heads)) return nullptr;
  const long path = PyLong_AsLong(patho);
  if (path == -1 && PyErr_Occurred()) return nullptr;
  return forward(table, n_layers, n_heads, *x, path, ws, y, is_static, false);
}

// head_forward(heads, x, path, ws, y)
PyObject* head_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return arity(n, 5) ? heads_call(a[0], a[1], a[2], a[3], a[4], false) : nullptr;
  END_HANDLE_TH_ERRORS
}

// head_forward_static(heads, x, path, y)
PyObject* head_forward_static(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  return arity(n, 4) ? heads_call(a[0], a[1], a[2], Py_None, a[3], true) : nullptr;
  END_HANDLE_TH_ERRORS
}

// dense_layer_forward(coef, x, ws, y)
PyObject* dense_layer_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 4)) return nullptr;
  const at::Tensor* coef = tensor_of(a[0], "coef");
  const at::Tensor* x = coef ? tensor_of(a[1], "x") : nullptr;
  if (!x || !check_floats(*coef, "coef")) return nullptr;
  if (!x->is_contiguous()) {
    PyErr_SetString(PyExc_AssertionError, "x: contiguous");
    return nullptr;
  }
  if (coef->dim() != 3 || x->dim() < 1) {
    PyErr_SetString(PyExc_ValueError, "coef: [in][out][10], x: [batch][in]");
    return nullptr;
  }
  const int64_t n_in = coef->size(0), n_out = coef->size(1), g = coef->size(2), B = x->size(0);
  Buffers b;
  size_t need = 0;
  if (a[2] == Py_None) {
    need = kan_dense_workspace_bytes((int32_t)n_in, (int32_t)n_out, B);
    if (need == (size_t)-1) return PyLong_FromLong(KAN_ERR_SHAPE);
  }
  if (!b.use_ws(a[2], need, *x) || !b.use_y(a[3], {B, n_out}, *x)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const float *cp = (const float*)coef->data_ptr(), *xp = (const float*)x->data_ptr();
  kan_status st;
  Py_BEGIN_ALLOW_THREADS
  st = kan_dense_layer_forward(cp, (int32_t)n_in, (int32_t)n_out, (int32_t)g, xp, B, (float*)b.y, b.ws, b.ws_bytes, stream);
  Py_END_ALLOW_THREADS
  return b.result(st);
  END_HANDLE_TH_ERRORS
}

// assign(coef, codebook, ws) -> (idx, gain, bias)
PyObject* assign(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 3)) return nullptr;
  const at::Tensor* coef = tensor_of(a[0], "coef");
  const at::Tensor* cb = coef ? tensor_of(a[1], "codebook") : nullptr;
  if (!cb || !check_floats(*coef, "coef") || !check_floats(*cb, "codebook")) return nullptr;
  if (coef->dim() != 3 || coef->size(2) != 10 || cb->dim() != 2 || cb->size(1) != 10) {
    PyErr_SetString(PyExc_AssertionError, "coef: [in][out][10], codebook: [K][10]");
    return nullptr;
  }
  const int64_t n_in = coef->size(0), n_out = coef->size(1), K = cb->size(0);
  const bool u16 = K <= 65536;
  at::Tensor idx = at::empty({n_in, n_out}, coef->options().dtype(u16 ? at::kShort : at::kInt));
  at::Tensor gain = at::empty({n_in, n_out}, coef->options()), bias = at::empty({n_in, n_out}, coef->options());
  Buffers b;
  size_t need = a[2] == Py_None ? kan_vq_assign_fast_workspace_bytes((int32_t)n_in, (int32_t)n_out, (int32_t)K) : 0;
  if (need == (size_t)-1) return PyLong_FromLong(KAN_ERR_SHAPE);
  if (!b.use_ws(a[2], need, *coef)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const float *cp = (const float*)coef->data_ptr(), *kp = (const float*)cb->data_ptr();
  void* ip = idx.data_ptr();
  float *gp = (float*)gain.data_ptr(), *bp = (float*)bias.data_ptr();
  kan_status st;
  Py_BEGIN_ALLOW_THREADS
  st = kan_vq_assign(cp, (int32_t)n_in, (int32_t)n_out, kp, (int32_t)K, u16 ? KAN_U16 : KAN_U32, ip, gp, bp, b.ws,
                     b.ws_bytes, stream);
  Py_END_ALLOW_THREADS
  if (st != KAN_OK) return PyLong_FromLong(st);
  PyObject* r = PyTuple_New(3);
  if (!r) return nullptr;
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(std::move(idx)));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(std::move(gain)));
  PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(std::move(bias)));
  return r;
  END_HANDLE_TH_ERRORS
}

// ---- the operators around the blocks of a language model -----------------------------------------------------------

bool g_poison = false;        // outputs of these calls start as NaN (KAN_POISON_OUTPUTS, see binding.py)

bool refuse(const char* what) {
  PyErr_SetString(PyExc_AssertionError, what);
  return false;
}

int float_code(at::ScalarType t) { return t == at::kFloat ? KAN_F32 : t == at::kHalf ? KAN_F16 : t == at::kBFloat16 ? KAN_BF16 : -1; }
int id_code(at::ScalarType t) { return t == at::kShort ? KAN_U16 : t == at::kInt ? KAN_U32 : t == at::kLong ? KAN_I64 : -1; }

// The current device, which the calls go to: every tensor has to be there.
struct Device {
  c10::Device dev = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice();

  bool holds(const at::Tensor& t, const char* what) const {
    if (t.device() != dev) {
      PyErr_Format(PyExc_AssertionError, "%s: not on the current device", what);
      return false;
    }
    if (!t.is_contiguous()) {
      PyErr_Format(PyExc_AssertionError, "%s: contiguous", what);
      return false;
    }
    return true;
  }
  // A tensor of float32, float16 or bfloat16; None is allowed where `optional` (the result is then empty).
  bool floats(PyObject* o, const char* what, bool optional, const at::Tensor** out) const {
    *out = nullptr;
    if (optional && o == Py_None) return true;
    const at::Tensor* t = tensor_of(o, what);
    if (!t || !holds(*t, what)) return false;
    if (float_code(t->scalar_type()) < 0) {
      PyErr_Format(PyExc_AssertionError, "%s: float32, float16 or bfloat16", what);
      return false;
    }
    *out = t;
    return true;
  }
  bool ids(PyObject* o, const char* what, const at::Tensor** out) const {
    const at::Tensor* t = tensor_of(o, what);
    if (!t || !holds(*t, what)) return false;
    if (id_code(t->scalar_type()) < 0) {
      PyErr_Format(PyExc_AssertionError, "%s: int16 (carrying uint16), int32 or int64", what);
      return false;
    }
    *out = t;
    return true;
  }
  // An output: the caller's tensor, which has to have this shape and type, or one of its own.
  bool output(PyObject* o, const char* what, at::IntArrayRef shape, at::ScalarType type, at::Tensor* out) const {
    if (o != Py_None) {
      const at::Tensor* t = tensor_of(o, what);
      if (!t || !holds(*t, what)) return false;
      if (t->sizes() != shape || t->scalar_type() != type) {
        PyErr_Format(PyExc_AssertionError, "%s: shape or dtype", what);
        return false;
      }
      *out = *t;
      return true;
    }
    const at::TensorOptions opt = at::TensorOptions().device(dev).dtype(type);
    *out = g_poison ? at::full(shape, NAN, opt) : at::empty(shape, opt);
    return true;
  }
  bool workspace(PyObject* o, size_t need, at::Tensor* out) const {
    if (o != Py_None) {
      const at::Tensor* t = tensor_of(o, "ws");
      if (!t || !holds(*t, "ws")) return false;
      *out = *t;
    } else if (need > 0 && need != (size_t)-1) {      // (a call with invalid sizes reports its status itself)
      *out = at::empty({(int64_t)need}, at::TensorOptions().device(dev).dtype(at::kByte));
    }
    return true;
  }
};

void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
void* ptr(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t bytes(const at::Tensor& t) { return t.defined() ? (size_t)t.nbytes() : 0; }

bool number(PyObject* o, float* out) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) return false;
  *out = (float)v;
  return true;
}

bool dtype_of(PyObject* o, at::ScalarType otherwise, at::ScalarType* out) {
  *out = otherwise;
  if (o == Py_None) return true;
  if (!THPDtype_Check(o)) return refuse("dtype: a torch.dtype");
  *out = reinterpret_cast<THPDtype*>(o)->scalar_type;
  return float_code(*out) >= 0 || refuse("dtype: float32, float16 or bfloat16");
}

// A size the C-ABI carries in 32 bits.
bool small(int64_t n) { return n <= INT32_MAX || refuse("a size past 2^31 - 1"); }

PyObject* wrapped(kan_status st, std::initializer_list<at::Tensor*> out) {
  if (st != KAN_OK) return PyLong_FromLong(st);
  if (out.size() == 1) return THPVariable_Wrap(std::move(**out.begin()));
  PyObject* r = PyTuple_New((Py_ssize_t)out.size());
  if (!r) return nullptr;
  Py_ssize_t i = 0;
  for (at::Tensor* t : out) {
    PyObject* v = Py_None;
    if (t->defined()) v = THPVariable_Wrap(std::move(*t));
    else Py_INCREF(v);
    PyTuple_SET_ITEM(r, i++, v);
  }
  return r;
}

// The C-ABI call, other Python threads running meanwhile.
template <class F>
kan_status unlocked(F&& f) {
  kan_status st;
  Py_BEGIN_ALLOW_THREADS
  st = f();
  Py_END_ALLOW_THREADS
  return st;
}

// lookup_forward(table, ids, scale, dtype, y)
PyObject* lookup_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 5)) return nullptr;
  const Device d;
  const at::Tensor *table, *ids;
  at::Tensor y;
  float scale;
  at::ScalarType type;
  if (!d.floats(a[0], "table", false, &table) || !d.ids(a[1], "ids", &ids) || !number(a[2], &scale) || !dtype_of(a[3], table->scalar_type(), &type)) return nullptr;
  if (table->dim() != 2) return refuse("table: [rows][columns]"), nullptr;
  if (!small(table->size(0)) || !small(table->size(1))) return nullptr;
  c10::SmallVector<int64_t, 8> shape(ids->sizes().begin(), ids->sizes().end());
  shape.push_back(table->size(1));
  if (a[4] != Py_None && a[3] == Py_None && THPVariable_Check(a[4])) type = THPVariable_Unpack(a[4]).scalar_type();
  if (float_code(type) < 0) return refuse("y: float32, float16 or bfloat16"), nullptr;
  if (!d.output(a[4], "y", shape, type, &y)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const kan_status st = unlocked([&] { return kan_lookup_forward(table->data_ptr(), float_code(table->scalar_type()), (int32_t)table->size(0), (int32_t)table->size(1), ids->data_ptr(),
                                           id_code(ids->scalar_type()), ids->numel(), scale, y.data_ptr(), float_code(type), stream); });
  return wrapped(st, {&y});
  END_HANDLE_TH_ERRORS
}

// lookup_backward(dy, ids, rows, scale, dtype, dtable, accumulate, ws)
PyObject* lookup_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 8)) return nullptr;
  const Device d;
  const at::Tensor *dy, *ids;
  at::Tensor dtable, ws;
  float scale;
  at::ScalarType type;
  if (!d.floats(a[0], "dy", false, &dy) || !d.ids(a[1], "ids", &ids) || !number(a[3], &scale) || !dtype_of(a[4], dy->scalar_type(), &type)) return nullptr;
  const long long rows = PyLong_AsLongLong(a[2]);
  if (rows == -1 && PyErr_Occurred()) return nullptr;
  const int accumulate = PyObject_IsTrue(a[6]);
  if (accumulate < 0) return nullptr;
  if (dy->dim() != ids->dim() + 1 || dy->sizes().slice(0, ids->dim()) != ids->sizes()) return refuse("dy: [shape of ids][columns]"), nullptr;
  const int64_t D = dy->size(dy->dim() - 1);
  if (rows < 1 || !small(rows) || !small(D)) return PyErr_Occurred() ? nullptr : PyLong_FromLong(KAN_ERR_SHAPE);
  if (accumulate && a[5] == Py_None) return refuse("accumulate: onto a dtable"), nullptr;
  if (a[5] != Py_None && a[4] == Py_None && THPVariable_Check(a[5])) type = THPVariable_Unpack(a[5]).scalar_type();
  if (float_code(type) < 0) return refuse("dtable: float32, float16 or bfloat16"), nullptr;
  if (!d.output(a[5], "dtable", {rows, D}, type, &dtable)) return nullptr;
  if (!d.workspace(a[7], a[7] == Py_None ? kan_lookup_backward_workspace_bytes((int32_t)rows, (int32_t)D, ids->numel()) : 0, &ws)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const kan_status st = unlocked([&] { return kan_lookup_backward(dy->data_ptr(), float_code(dy->scalar_type()), ids->data_ptr(), id_code(ids->scalar_type()), ids->numel(),
                                            (int32_t)rows, (int32_t)D, scale, dtable.data_ptr(), float_code(type), accumulate, ptr(ws), bytes(ws), stream); });
  return wrapped(st, {&dtable});
  END_HANDLE_TH_ERRORS
}

// The weights, scale and eps of a pair of norms; x: any tensor of the stream.
bool read_norm(const Device& d, PyObject* w_after, PyObject* w_before, PyObject* scale, PyObject* eps, const at::Tensor& x, at::ScalarType block,
               kan_block_norm* b, const at::Tensor** wa, const at::Tensor** wb) {
  if (!d.floats(w_after, "w_after", true, wa) || !d.floats(w_before, "w_before", true, wb)) return false;
  if (x.dim() < 1) return refuse("x: [...][columns]");
  const int64_t D = x.size(x.dim() - 1);
  if (!small(D)) return false;
  for (const at::Tensor* w : {*wa, *wb})
    if (w && (w->dim() != 1 || w->size(0) != D)) return refuse("w_after, w_before: [columns]");
  if (*wa && *wb && (*wa)->scalar_type() != (*wb)->scalar_type()) return refuse("w_after, w_before: one dtype");
  *b = {};
  b->D = (int32_t)D;
  b->stream_dtype = float_code(x.scalar_type());
  b->block_dtype = float_code(block);
  b->weight_dtype = *wa ? float_code((*wa)->scalar_type()) : *wb ? float_code((*wb)->scalar_type()) : KAN_F32;
  b->w_before = ptr(*wb);
  b->w_after = ptr(*wa);
  return number(scale, &b->scale) && number(eps, &b->eps);
}

bool same(const at::Tensor* t, const at::Tensor& shape, at::ScalarType type, const char* what) {
  if (!t || (t->sizes() == shape.sizes() && t->scalar_type() == type)) return true;
  PyErr_Format(PyExc_AssertionError, "%s: shape or dtype", what);
  return false;
}

// block_norm_forward(x, v, gate, w_after, w_before, scale, eps, dtype, want_u, y, u) -> (y, u)
PyObject* block_norm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 11)) return nullptr;
  const Device d;
  const at::Tensor *x, *v, *gate, *wa, *wb;
  at::Tensor y, u;
  at::ScalarType block;
  kan_block_norm b;
  if (!d.floats(a[0], "x", false, &x) || !d.floats(a[1], "v", true, &v) || !d.floats(a[2], "gate", true, &gate) ||
      !dtype_of(a[7], v ? v->scalar_type() : x->scalar_type(), &block) || !read_norm(d, a[3], a[4], a[5], a[6], *x, block, &b, &wa, &wb) ||
      !same(v, *x, block, "v") || !same(gate, *x, block, "gate"))
    return nullptr;
  const int want_u = PyObject_IsTrue(a[8]);
  if (want_u < 0) return nullptr;
  if (!v && (gate || a[9] != Py_None)) return refuse("gate, y: only behind a block (v)"), nullptr;
  if (!v && !want_u) return refuse("neither a block's output v nor a norm in front of one"), nullptr;
  if (!want_u && a[10] != Py_None) return refuse("u: not wanted"), nullptr;
  if (v && !d.output(a[9], "y", x->sizes(), x->scalar_type(), &y)) return nullptr;
  if (want_u && !d.output(a[10], "u", x->sizes(), block, &u)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const kan_status st = unlocked([&] { return kan_block_norm_forward(&b, x->data_ptr(), ptr(v), ptr(gate), b.D ? x->numel() / b.D : 0, ptr(y), ptr(u), stream); });
  return wrapped(st, {&y, &u});
  END_HANDLE_TH_ERRORS
}

// block_norm_backward(y, dy, du, v, gate, w_after, w_before, scale, eps, ws) -> (dx, dv, dgate, dw_before, dw_after)
PyObject* block_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 10)) return nullptr;
  const Device d;
  const at::Tensor *y, *dy, *du, *v, *gate, *wa, *wb;
  at::Tensor dx, dv, dgate, dwb, dwa, ws;
  kan_block_norm b;
  if (!d.floats(a[0], "y", false, &y) || !d.floats(a[1], "dy", true, &dy) || !d.floats(a[2], "du", true, &du) || !d.floats(a[3], "v", true, &v) ||
      !d.floats(a[4], "gate", true, &gate))
    return nullptr;
  const at::ScalarType stream_type = y->scalar_type(), block = du ? du->scalar_type() : v ? v->scalar_type() : stream_type;
  if (!read_norm(d, a[5], a[6], a[7], a[8], *y, block, &b, &wa, &wb) || !same(dy, *y, stream_type, "dy") || !same(du, *y, block, "du") ||
      !same(v, *y, block, "v") || !same(gate, *y, block, "gate"))
    return nullptr;
  if (!dy && !du) return refuse("neither dy nor du"), nullptr;
  if (!v && gate) return refuse("gate: only behind a block (v)"), nullptr;
  if (!d.output(Py_None, "dx", y->sizes(), stream_type, &dx)) return nullptr;
  if (v && !d.output(Py_None, "dv", y->sizes(), block, &dv)) return nullptr;
  if (gate && !d.output(Py_None, "dgate", y->sizes(), block, &dgate)) return nullptr;
  if (wb && du && !d.output(Py_None, "dw_before", wb->sizes(), wb->scalar_type(), &dwb)) return nullptr;
  if (wa && v && !d.output(Py_None, "dw_after", wa->sizes(), wa->scalar_type(), &dwa)) return nullptr;
  const int64_t N = b.D ? y->numel() / b.D : 0;
  if (!d.workspace(a[9], a[9] == Py_None ? kan_block_norm_backward_workspace_bytes(&b, N) : 0, &ws)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const kan_status st = unlocked([&] { return kan_block_norm_backward(&b, y->data_ptr(), ptr(dy), ptr(du), ptr(v), ptr(gate), N, dx.data_ptr(), ptr(dv), ptr(dgate), ptr(dwb),
                                                ptr(dwa), ptr(ws), bytes(ws), stream); });
  return wrapped(st, {&dx, &dv, &dgate, &dwb, &dwa});
  END_HANDLE_TH_ERRORS
}

// h: [...][D], table: [V][D] of the same dtype, targets: [...]
bool read_vocab(const Device& d, PyObject* ho, PyObject* to, PyObject* targetso, const at::Tensor** h, const at::Tensor** table, const at::Tensor** targets) {
  if (!d.floats(ho, "h", false, h) || !d.floats(to, "table", false, table) || !d.ids(targetso, "targets", targets)) return false;
  if ((*table)->dim() != 2 || (*h)->dim() < 1 || (*h)->size((*h)->dim() - 1) != (*table)->size(1) || (*h)->scalar_type() != (*table)->scalar_type())
    return refuse("h: [...][columns], table: [rows][columns], one dtype");
  if ((*targets)->sizes() != (*h)->sizes().slice(0, (*h)->dim() - 1)) return refuse("targets: a target for every row of h");
  return small((*table)->size(0)) && small((*table)->size(1));
}

// vocab_loss_forward(h, table, targets, scale, loss, lse, ws) -> (loss, lse)
PyObject* vocab_loss_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 7)) return nullptr;
  const Device d;
  const at::Tensor *h, *table, *targets;
  at::Tensor loss, lse, ws;
  float scale;
  if (!read_vocab(d, a[0], a[1], a[2], &h, &table, &targets) || !number(a[3], &scale) || !d.output(a[4], "loss", targets->sizes(), at::kFloat, &loss) ||
      !d.output(a[5], "lse", targets->sizes(), at::kFloat, &lse))
    return nullptr;
  const int dtype = float_code(h->scalar_type());
  const int32_t V = (int32_t)table->size(0), D = (int32_t)table->size(1);
  if (!d.workspace(a[6], a[6] == Py_None ? kan_vocab_loss_workspace_bytes(targets->numel(), V, D, dtype, 0) : 0, &ws)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const kan_status st = unlocked([&] { return kan_vocab_loss_forward(h->data_ptr(), table->data_ptr(), dtype, targets->numel(), V, D, targets->data_ptr(),
                                               id_code(targets->scalar_type()), scale, (float*)loss.data_ptr(), (float*)lse.data_ptr(), ptr(ws), bytes(ws), stream); });
  return wrapped(st, {&loss, &lse});
  END_HANDLE_TH_ERRORS
}

// vocab_loss_backward(h, table, targets, lse, dloss, scale, dh, dtable, accumulate, ws) -> (dh, dtable)
PyObject* vocab_loss_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (!arity(n, 10)) return nullptr;
  const Device d;
  const at::Tensor *h, *table, *targets, *lse, *dloss;
  at::Tensor dh, dtable, ws;
  float scale;
  if (!read_vocab(d, a[0], a[1], a[2], &h, &table, &targets) || !d.floats(a[3], "lse", false, &lse) || !d.floats(a[4], "dloss", false, &dloss) ||
      !same(lse, *targets, at::kFloat, "lse") || !same(dloss, *targets, at::kFloat, "dloss") || !number(a[5], &scale))
    return nullptr;
  const int accumulate = PyObject_IsTrue(a[8]);
  if (accumulate < 0) return nullptr;
  if (accumulate && a[7] == Py_None) return refuse("accumulate: onto a dtable"), nullptr;
  if (!d.output(a[6], "dh", h->sizes(), h->scalar_type(), &dh) || !d.output(a[7], "dtable", table->sizes(), table->scalar_type(), &dtable)) return nullptr;
  const int dtype = float_code(h->scalar_type());
  const int32_t V = (int32_t)table->size(0), D = (int32_t)table->size(1);
  if (!d.workspace(a[9], a[9] == Py_None ? kan_vocab_loss_workspace_bytes(targets->numel(), V, D, dtype, 1) : 0, &ws)) return nullptr;
  void* stream;
  if (!current_stream(&stream)) return nullptr;
  const kan_status st = unlocked([&] { return kan_vocab_loss_backward(h->data_ptr(), table->data_ptr(), dtype, targets->numel(), V, D, targets->data_ptr(),
                                                id_code(targets->scalar_type()), scale, (const float*)lse->data_ptr(), (const float*)dloss->data_ptr(),
                                                dh.data_ptr(), dtable.data_ptr(), accumulate, ptr(ws), bytes(ws), stream); });
  return wrapped(st, {&dh, &dtable});
  END_HANDLE_TH_ERRORS
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(F)), METH_FASTCALL, nullptr};
}

PyMethodDef g_methods[] = {method<layer_forward>("layer_forward"),
                           method<head_forward>("head_forward"),
                           method<head_forward_static>("head_forward_static"),
                           method<dense_layer_forward>("dense_layer_forward"),
                           method<assign>("assign"),
                           method<lookup_forward>("lookup_forward"),
                           method<lookup_backward>("lookup_backward"),
                           method<block_norm_forward>("block_norm_forward"),
                           method<block_norm_backward>("block_norm_backward"),
                           method<vocab_loss_forward>("vocab_loss_forward"),
                           method<vocab_loss_backward>("vocab_loss_backward"),
                           {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_kan_host", "Per-request entry points of the binding.", -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kan_host(void) {
  const char* const poison = getenv("KAN_POISON_OUTPUTS");
  g_poison = poison && *poison && strcmp(poison, "0") != 0;
  g_desc_name = PyUnicode_InternFromString("desc");
  PyObject* c = PyImport_ImportModule("torch._C");
  if (!g_desc_name || !c) return nullptr;
  g_raw_stream = PyObject_GetAttrString(c, "_cuda_getCurrentRawStream");
  Py_DECREF(c);
  if (!g_raw_stream) return nullptr;
  return PyModule_Create(&g_module);
}
