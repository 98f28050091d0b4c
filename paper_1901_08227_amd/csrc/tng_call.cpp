// The hot calls of binding.py without a trip through ctypes: an argument check and the call of a C entry point, in one
// extension function.  What bounds a small call is the host: of the 11.5 us that encode + decode of 4 x 25000 gradients took
// back to back, 8.5 were kernels; a pass through the checks in Python and ctypes is 0.5 to 0.7 us a tensor.
//
//   call(address, handle, iter, kinds, d, M, words, tensor, ...) -> status, or None
//
// address: of the entry point; kinds: a letter per tensor, d float32[d], g float32[M d], c int32[M words], s float32[M], behind a
// '-' for an entry point that takes no iteration number (iter is then not looked at).  None says that an argument is not a plain
// case (no tensor, another type, too short, a tensor subclass other than Parameter or a wrapper without storage, an iteration that
// is no int): nothing was called, and the caller goes the way through ctypes, which raises what there is to raise.
//
//   layer(address, address of the call that sizes its scratch, stream, kinds, argument, ...) -> status, or None
//
// the same for the calls on layers: kinds has a letter per argument, m a matrix of numbers ([rows, cols] or [M, rows, cols]), i one of codes,
// d the five fields of tng_drop in a tuple, and float32 vectors by the last matrix before them: r workers * rows, n rows, c cols long.  A w
// (W) at the end takes no argument: scratch, as large as is said of the first matrix (of the first two and the last), from torch.  Nor
// does an o (p): a matrix like the first (with a column for each row of the last before it), from torch; that tensor is what is returned
// where the call succeeds.
//
//   linear(addresses, stream, x, drop, codes, scales, bias) -> (y, scales, turned codes)
//   linear_grad(addresses, stream, dy, scales, turned codes, weights' scales, weights' turned codes, drop, x, (seed, iter, site), out)
//     -> (dx, dw, db)
//
// whole layers in training, what they put in between from torch: None as above, or the status of a call that refused.  addresses: a tuple.
#include <Python.h>

#include <algorithm>
#include <cstring>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/util/SmallVector.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/tng.h"

namespace {

constexpr int kFixed = 7, kMaxTensors = 6;

// True if obj is a plain device tensor of that type and at least n elements; *p is its address (null for None).
bool device_address(PyObject* obj, char kind, int64_t d, int64_t M, int64_t words, void** p) {
  if (obj == Py_None) {
    *p = nullptr;
    return true;
  }
  if (!THPVariable_CheckExact(obj)) return false;
  const at::Tensor& t = THPVariable_Unpack(obj);
  if (!t.defined() || !t.has_storage() || !t.is_cuda() || t.layout() != at::kStrided || !t.is_contiguous()) return false;
  if (t.scalar_type() != (kind == 'c' ? at::kInt : at::kFloat)) return false;
  const int64_t n = kind == 'd' ? d : kind == 'g' ? M * d : kind == 'c' ? M * words : M;
  if (t.numel() < n) return false;
  *p = t.data_ptr();
  return true;
}

template <typename... P>
int enter(uintptr_t f, void* h, bool with_iter, uint32_t iter, P... p) {
  if (with_iter) return reinterpret_cast<int (*)(void*, uint32_t, P...)>(f)(h, iter, p...);
  return reinterpret_cast<int (*)(void*, P...)>(f)(h, p...);
}

PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  const Py_ssize_t n = nargs - kFixed;
  const char* kinds = nullptr;
  if (n < 2 || n > kMaxTensors || !PyUnicode_Check(args[3]) || (kinds = PyUnicode_AsUTF8(args[3])) == nullptr ||
      PyUnicode_GET_LENGTH(args[3]) != n + (kinds[0] == '-')) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "call: a letter per tensor, 2 to 6 tensors");
    return nullptr;
  }
  const bool with_iter = kinds[0] != '-';
  if (!with_iter) ++kinds;
  // (anything but a plain int as handle or iteration, None too, goes through ctypes, which converts or refuses it)
  if (!PyLong_CheckExact(args[1]) || (with_iter && !PyLong_CheckExact(args[2]))) Py_RETURN_NONE;
  const uintptr_t f = (uintptr_t)PyLong_AsUnsignedLongLong(args[0]);
  void* h = reinterpret_cast<void*>((uintptr_t)PyLong_AsUnsignedLongLong(args[1]));
  const uint32_t iter = with_iter ? (uint32_t)PyLong_AsUnsignedLongMask(args[2]) : 0u;  // (as ctypes does)
  const int64_t d = PyLong_AsLongLong(args[4]), M = PyLong_AsLongLong(args[5]), words = PyLong_AsLongLong(args[6]);
  if (PyErr_Occurred()) return nullptr;
  void* p[kMaxTensors] = {};
  try {
    for (Py_ssize_t i = 0; i < n; ++i)
      if (!device_address(args[kFixed + i], kinds[i], d, M, words, &p[i])) Py_RETURN_NONE;
  } catch (const std::exception&) {  // (an address that cannot be had: ctypes' way says why)
    Py_RETURN_NONE;
  }
  int status = -1;
  Py_BEGIN_ALLOW_THREADS
  switch (n) {
    case 2: status = enter(f, h, with_iter, iter, p[0], p[1]); break;
    case 3: status = enter(f, h, with_iter, iter, p[0], p[1], p[2]); break;
    case 4: status = enter(f, h, with_iter, iter, p[0], p[1], p[2], p[3]); break;
    case 5: status = enter(f, h, with_iter, iter, p[0], p[1], p[2], p[3], p[4]); break;
    default: status = enter(f, h, with_iter, iter, p[0], p[1], p[2], p[3], p[4], p[5]); break;
  }
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

using Shape = c10::SmallVector<int64_t, 4>;

// [M, rows, cols], without the M where x had none.
Shape shape_like(const at::Tensor& x, int64_t rows, int64_t cols) {
  Shape s;
  if (x.dim() == 3) s.push_back(x.size(0));
  s.push_back(rows);
  s.push_back(cols);
  return s;
}

// A matrix of numbers of x's type (or float32), and its tng_matrix.
at::Tensor numbers(const at::Tensor& x, int64_t rows, int64_t cols, at::ScalarType type, tng_matrix* m) {
  const at::Tensor t = at::empty(shape_like(x, rows, cols), x.options().dtype(type));
  *m = tng_matrix{t.data_ptr(), type == at::kFloat ? TNG_TYPE_F32 : type == at::kHalf ? TNG_TYPE_F16 : TNG_TYPE_BF16,
                  x.dim() == 3 ? (uint32_t)x.size(0) : 1u, (uint64_t)rows, (uint64_t)cols, (uint64_t)cols, (uint64_t)(rows * cols)};
  return t;
}

constexpr int kLayerFixed = 4, kLayerMost = 16;

// One argument of a layer call as the 64 bits that the entry point takes.
struct LayerCall {
  tng_matrix matrix[8];
  int matrices = 0;
  tng_drop drop;
  c10::Device device{c10::kCPU};
  bool have_device = false;
  PyObject* first = nullptr;  // the first matrix

  bool same_device(const at::Tensor& t) {
    if (!have_device) {
      device = t.device();
      have_device = true;
    }
    return t.device() == device;
  }

  bool tensor(PyObject* obj, at::Tensor* t) {
    if (!THPVariable_CheckExact(obj)) return false;
    *t = THPVariable_Unpack(obj);
    return t->defined() && t->has_storage() && t->is_cuda() && t->layout() == at::kStrided && same_device(*t);
  }

  bool as_matrix(PyObject* obj, bool codes, uintptr_t* out) {
    at::Tensor t;
    if (matrices == 8 || !tensor(obj, &t)) return false;
    tng_matrix& m = matrix[matrices];
    switch (t.scalar_type()) {
      case at::kFloat: m.type = TNG_TYPE_F32; break;
      case at::kBFloat16: m.type = TNG_TYPE_BF16; break;
      case at::kHalf: m.type = TNG_TYPE_F16; break;
      case at::kChar: m.type = TNG_TYPE_I8; break;
      default: return false;
    }
    if ((m.type == TNG_TYPE_I8) != codes) return false;
    const int64_t dim = t.dim();
    if (dim != 2 && dim != 3) return false;
    const auto sizes = t.sizes();
    const auto strides = t.strides();
    if (strides[dim - 1] != 1 && sizes[dim - 1] > 1) return false;
    if (dim == 3 && (sizes[0] < 1 || sizes[0] > 65535)) return false;
    m.data = t.data_ptr();
    m.workers = dim == 3 ? (uint32_t)sizes[0] : 1u;
    m.rows = (uint64_t)sizes[dim - 2];
    m.cols = (uint64_t)sizes[dim - 1];
    m.ld = (uint64_t)strides[dim - 2];
    m.pitch = dim == 3 ? (uint64_t)strides[0] : 0u;
    if (matrices++ == 0) first = obj;
    *out = reinterpret_cast<uintptr_t>(&m);
    return true;
  }

  bool as_vector(PyObject* obj, char kind, uintptr_t* out) {
    at::Tensor t;
    if (matrices == 0 || !tensor(obj, &t) || t.scalar_type() != at::kFloat || !t.is_contiguous()) return false;
    const tng_matrix& m = matrix[matrices - 1];
    if ((uint64_t)t.numel() != (kind == 'r' ? m.workers * m.rows : kind == 'n' ? m.rows : m.cols)) return false;
    *out = reinterpret_cast<uintptr_t>(t.data_ptr());
    return true;
  }

  bool as_drop(PyObject* obj, uintptr_t* out) {
    if (!PyTuple_Check(obj) || PyTuple_GET_SIZE(obj) != 5) return false;
    PyObject* f[5];
    for (int i = 0; i < 5; ++i) f[i] = PyTuple_GET_ITEM(obj, i);
    if (!PyLong_CheckExact(f[0]) || !PyLong_CheckExact(f[1]) || !PyLong_CheckExact(f[2]) || !PyFloat_CheckExact(f[3]) || !PyBool_Check(f[4]))
      return false;
    drop.seed = PyLong_AsUnsignedLongLongMask(f[0]);
    drop.iter = (uint32_t)PyLong_AsUnsignedLongMask(f[1]);
    int overflow = 0;
    const long long site = PyLong_AsLongLongAndOverflow(f[2], &overflow);
    if (overflow != 0 || site < 0 || site > 0xFFFFFFFFll) return false;
    drop.site = (uint32_t)site;
    drop.p = (float)PyFloat_AS_DOUBLE(f[3]);
    drop.relu = f[4] == Py_True;
    *out = reinterpret_cast<uintptr_t>(&drop);
    return true;
  }
};

template <size_t... I>
int enter_layer(uintptr_t f, const uintptr_t* a, std::index_sequence<I...>) {
  return reinterpret_cast<int (*)(decltype((void)I, uintptr_t{})...)>(f)(a[I]...);
}

PyObject* layer(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  const char* kinds = nullptr;
  if (nargs < kLayerFixed || !PyUnicode_Check(args[3]) || (kinds = PyUnicode_AsUTF8(args[3])) == nullptr) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "layer: addresses, a stream, kinds and their arguments");
    return nullptr;
  }
  const Py_ssize_t letters = PyUnicode_GET_LENGTH(args[3]);
  const bool scratch = letters > 0 && (kinds[letters - 1] == 'w' || kinds[letters - 1] == 'W');
  Py_ssize_t made = 0;  // without an argument
  for (Py_ssize_t i = 0; i < letters; ++i) made += strchr("wWop", kinds[i]) != nullptr;
  if (nargs != kLayerFixed + letters - made || letters > kLayerMost - 3) {
    PyErr_SetString(PyExc_TypeError, "layer: an argument per letter");
    return nullptr;
  }
  const uintptr_t f = (uintptr_t)PyLong_AsUnsignedLongLong(args[0]), sizes = (uintptr_t)PyLong_AsUnsignedLongLong(args[1]);
  uintptr_t a[kLayerMost] = {(uintptr_t)PyLong_AsUnsignedLongLong(args[2])};
  if (PyErr_Occurred()) return nullptr;
  LayerCall c;
  int n = 1, status = -1;
  try {
    at::Tensor out;
    PyObject* const* next = args + kLayerFixed;
    for (Py_ssize_t i = 0; i < letters - scratch; ++i, ++n) {
      if (kinds[i] == 'o' || kinds[i] == 'p') {
        if (c.matrices == 0 || c.matrices == 8 || c.first == nullptr) Py_RETURN_NONE;
        const tng_matrix& m = c.matrix[0];
        const at::Tensor& like = THPVariable_Unpack(c.first);
        out = numbers(like, (int64_t)m.rows, (int64_t)(kinds[i] == 'o' ? m.cols : c.matrix[c.matrices - 1].rows), like.scalar_type(),
                      &c.matrix[c.matrices]);
        a[n] = reinterpret_cast<uintptr_t>(&c.matrix[c.matrices++]);
        continue;
      }
      PyObject* obj = *next++;
      if (obj == Py_None) {
        a[n] = 0;
        continue;
      }
      const char k = kinds[i];
      const bool plain = k == 'd' ? c.as_drop(obj, &a[n]) : k == 'm' || k == 'i' ? c.as_matrix(obj, k == 'i', &a[n]) : c.as_vector(obj, k, &a[n]);
      if (!plain) Py_RETURN_NONE;
    }
    at::Tensor held;
    if (scratch) {
      if (c.matrices < (kinds[letters - 1] == 'w' ? 1 : 3)) Py_RETURN_NONE;
      const size_t bytes = kinds[letters - 1] == 'w'
                               ? reinterpret_cast<size_t (*)(const tng_matrix*)>(sizes)(&c.matrix[0])
                               : reinterpret_cast<size_t (*)(const tng_matrix*, const tng_matrix*, const tng_matrix*)>(sizes)(
                                     &c.matrix[0], &c.matrix[1], &c.matrix[c.matrices - 1]);
      if (bytes == 0) Py_RETURN_NONE;  // (refused: ctypes' way says what by)
      held = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(c.device));
      a[n++] = reinterpret_cast<uintptr_t>(held.data_ptr());
      a[n++] = bytes;
    }
    Py_BEGIN_ALLOW_THREADS
    switch (n) {
      case 5: status = enter_layer(f, a, std::make_index_sequence<5>{}); break;
      case 6: status = enter_layer(f, a, std::make_index_sequence<6>{}); break;
      case 9: status = enter_layer(f, a, std::make_index_sequence<9>{}); break;
      case 11: status = enter_layer(f, a, std::make_index_sequence<11>{}); break;
      case 12: status = enter_layer(f, a, std::make_index_sequence<12>{}); break;
      default: break;
    }
    Py_END_ALLOW_THREADS
    if (status == 0 && out.defined()) return THPVariable_Wrap(out);
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
  if (status < 0) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}

// ---- whole layers

using QuantizeRows = int (*)(uintptr_t, const tng_drop*, const tng_matrix*, const tng_matrix*, float*, const tng_matrix*);
using QuantizeGrad = int (*)(uintptr_t, const tng_drop*, const tng_matrix*, const float*, const float*, const tng_matrix*, float*,
                             const tng_matrix*, float*, float*, void*, size_t);
using GradBytes = size_t (*)(const tng_matrix*);
using Product = int (*)(uintptr_t, const tng_matrix*, const float*, const tng_matrix*, const float*, const float*, const tng_drop*,
                        const tng_matrix*, const tng_matrix*, void*, size_t);
using ProductBytes = size_t (*)(const tng_matrix*, const tng_matrix*, const tng_matrix*);

struct Entries {
  QuantizeRows quantize_rows;
  QuantizeGrad quantize_grad;
  GradBytes grad_bytes;
  Product product;
  ProductBytes product_bytes;
};

bool entries_of(PyObject* obj, Entries* e) {
  if (!PyTuple_Check(obj) || PyTuple_GET_SIZE(obj) != 5) return false;
  uintptr_t a[5];
  for (int i = 0; i < 5; ++i) a[i] = (uintptr_t)PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(obj, i));
  e->quantize_rows = reinterpret_cast<QuantizeRows>(a[0]);
  e->quantize_grad = reinterpret_cast<QuantizeGrad>(a[1]);
  e->grad_bytes = reinterpret_cast<GradBytes>(a[2]);
  e->product = reinterpret_cast<Product>(a[3]);
  e->product_bytes = reinterpret_cast<ProductBytes>(a[4]);
  return !PyErr_Occurred();
}

// Codes whose rows begin 16 bytes apart, and their matrix.
at::Tensor codes(const at::Tensor& x, int64_t rows, int64_t cols, tng_matrix* m) {
  const int64_t ld = (cols + 15) / 16 * 16;
  const at::Tensor t = at::empty(shape_like(x, rows, ld), x.options().dtype(at::kChar));
  *m = tng_matrix{t.data_ptr(), TNG_TYPE_I8, x.dim() == 3 ? (uint32_t)x.size(0) : 1u, (uint64_t)rows, (uint64_t)cols, (uint64_t)ld,
                  (uint64_t)(rows * ld)};
  return ld == cols ? t : t.narrow(-1, 0, cols);
}

// A float32 vector: a row of each worker's.
at::Tensor floats(const at::Tensor& x, int64_t n) {
  Shape s;
  if (x.dim() == 3) s.push_back(x.size(0));
  s.push_back(n);
  return at::empty(s, x.options().dtype(at::kFloat));
}

at::Tensor bytes_of(const at::Tensor& x, size_t n) { return at::empty({(int64_t)n}, x.options().dtype(at::kByte)); }

PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  Entries e;
  if (nargs != 7 || !entries_of(args[0], &e)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "linear: addresses, stream, x, drop, codes, scales, bias");
    return nullptr;
  }
  const uintptr_t stream = (uintptr_t)PyLong_AsUnsignedLongLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  try {
    LayerCall c;
    uintptr_t mx, mw, drop = 0, scales, bias = 0;
    if (!c.as_matrix(args[2], false, &mx) || (args[3] != Py_None && !c.as_drop(args[3], &drop)) || !c.as_matrix(args[4], true, &mw) ||
        !c.as_vector(args[5], 'r', &scales) || (args[6] != Py_None && !c.as_vector(args[6], 'n', &bias)))
      Py_RETURN_NONE;
    const tng_matrix x = c.matrix[0], w = c.matrix[1];
    if (w.cols != x.cols || w.workers != 1) Py_RETURN_NONE;
    const at::Tensor& tx = THPVariable_Unpack(args[2]);
    tng_matrix q, qt, y;
    const at::Tensor tq = codes(tx, x.rows, x.cols, &q), tqt = codes(tx, x.cols, x.rows, &qt), ts = floats(tx, x.rows);
    const at::Tensor ty = numbers(tx, x.rows, w.rows, tx.scalar_type(), &y);
    const size_t bytes = e.product_bytes(&q, &w, &y);
    if (bytes == 0) Py_RETURN_NONE;
    const at::Tensor scratch = bytes_of(tx, bytes);
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = e.quantize_rows(stream, reinterpret_cast<const tng_drop*>(drop), &x, &q, ts.data_ptr<float>(), &qt);
    if (status == 0)
      status = e.product(stream, &q, ts.data_ptr<float>(), &w, reinterpret_cast<const float*>(scales), reinterpret_cast<const float*>(bias),
                         nullptr, nullptr, &y, scratch.data_ptr(), bytes);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyLong_FromLong(status);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(ty), THPVariable_Wrap(ts), THPVariable_Wrap(tqt));
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

PyObject* linear_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  Entries e;
  if (nargs != 11 || !entries_of(args[0], &e)) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "linear_grad: addresses, stream, dy, scales, turned codes, those of the weights, drop, x, key, out");
    return nullptr;
  }
  const uintptr_t stream = (uintptr_t)PyLong_AsUnsignedLongLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  try {
    LayerCall c, k;
    uintptr_t at, row_scale, col_scale, drop = 0, gate = 0, key;
    // in the order in which a vector's length goes by the matrix before it
    if (!c.as_matrix(args[2], false, &at) || !c.as_vector(args[3], 'r', &row_scale) || !c.as_vector(args[5], 'c', &col_scale) ||
        !c.as_matrix(args[4], true, &at) || !c.as_matrix(args[6], true, &at) || (args[7] != Py_None && !c.as_drop(args[7], &drop)) ||
        (args[8] != Py_None && !c.as_matrix(args[8], false, &gate)) || !k.as_drop(args[9], &key))
      Py_RETURN_NONE;
    const tng_matrix dy = c.matrix[0], xt = c.matrix[1], wt = c.matrix[2];
    if (xt.cols != dy.rows || xt.workers != dy.workers || wt.cols != dy.cols || wt.rows != xt.rows || wt.workers != 1) Py_RETURN_NONE;
    const at::Tensor& ty = THPVariable_Unpack(args[2]);
    tng_matrix q, qt, dx, dw;
    at::Tensor tdw;
    if (args[10] == Py_None) {
      tdw = numbers(ty, dy.cols, xt.rows, at::kFloat, &dw);
    } else {
      if (!c.as_matrix(args[10], false, &at)) Py_RETURN_NONE;
      dw = *reinterpret_cast<const tng_matrix*>(at);
      tdw = THPVariable_Unpack(args[10]);
      if (dw.type != TNG_TYPE_F32 || dw.rows != dy.cols || dw.cols != xt.rows || tdw.dim() != ty.dim()) Py_RETURN_NONE;
    }
    const at::Tensor tq = codes(ty, dy.rows, dy.cols, &q), tqt = codes(ty, dy.cols, dy.rows, &qt);
    const at::Tensor tqs = floats(ty, dy.rows), tqts = floats(ty, dy.cols), tdb = floats(ty, dy.cols);
    const at::Tensor tdx = numbers(ty, dy.rows, xt.rows, ty.scalar_type(), &dx);
    // one scratch for the three calls, which follow each other on the stream
    const size_t first = e.grad_bytes(&dy), second = e.product_bytes(&q, &wt, &dx), third = e.product_bytes(&qt, &xt, &dw);
    if (first == 0 || second == 0 || third == 0) Py_RETURN_NONE;
    const size_t bytes = std::max(first, std::max(second, third));
    const at::Tensor scratch = bytes_of(ty, bytes);
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = e.quantize_grad(stream, reinterpret_cast<const tng_drop*>(key), &dy, reinterpret_cast<const float*>(col_scale),
                             reinterpret_cast<const float*>(row_scale), &q, tqs.data_ptr<float>(), &qt, tqts.data_ptr<float>(),
                             tdb.data_ptr<float>(), scratch.data_ptr(), bytes);
    if (status == 0)
      status = e.product(stream, &q, tqs.data_ptr<float>(), &wt, nullptr, nullptr, reinterpret_cast<const tng_drop*>(drop),
                         reinterpret_cast<const tng_matrix*>(gate), &dx, scratch.data_ptr(), bytes);
    if (status == 0)
      status = e.product(stream, &qt, tqts.data_ptr<float>(), &xt, nullptr, nullptr, nullptr, nullptr, &dw, scratch.data_ptr(), bytes);
    Py_END_ALLOW_THREADS
    if (status != 0) return PyLong_FromLong(status);
    return Py_BuildValue("(NNN)", THPVariable_Wrap(tdx), THPVariable_Wrap(tdw), THPVariable_Wrap(tdb));
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
}

PyMethodDef methods[] = {
    {"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL, nullptr},
    {"layer", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer)), METH_FASTCALL, nullptr},
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear)), METH_FASTCALL, nullptr},
    {"linear_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(linear_grad)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "tng_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the torch and Python that this was compiled for (the binding uses it with no other).
PyMODINIT_FUNC PyInit_tng_call() {
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "built_for", TNG_BUILT_FOR) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
