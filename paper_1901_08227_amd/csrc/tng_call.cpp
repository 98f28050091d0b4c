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
// (W) at the end takes no argument: scratch, as large as is said of the first matrix (of the first two and the last), from torch.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
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

constexpr int kLayerFixed = 4, kLayerMost = 16;

// One argument of a layer call as the 64 bits that the entry point takes.
struct LayerCall {
  tng_matrix matrix[8];
  int matrices = 0;
  tng_drop drop;
  c10::Device device{c10::kCPU};
  bool have_device = false;

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
    ++matrices;
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
  if (nargs != kLayerFixed + letters - scratch || letters > kLayerMost - 3) {
    PyErr_SetString(PyExc_TypeError, "layer: an argument per letter");
    return nullptr;
  }
  const uintptr_t f = (uintptr_t)PyLong_AsUnsignedLongLong(args[0]), sizes = (uintptr_t)PyLong_AsUnsignedLongLong(args[1]);
  uintptr_t a[kLayerMost] = {(uintptr_t)PyLong_AsUnsignedLongLong(args[2])};
  if (PyErr_Occurred()) return nullptr;
  LayerCall c;
  int n = 1, status = -1;
  try {
    for (Py_ssize_t i = 0; i < letters - scratch; ++i, ++n) {
      PyObject* obj = args[kLayerFixed + i];
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
      case 11: status = enter_layer(f, a, std::make_index_sequence<11>{}); break;
      case 12: status = enter_layer(f, a, std::make_index_sequence<12>{}); break;
      default: break;
    }
    Py_END_ALLOW_THREADS
  } catch (const std::exception&) {
    Py_RETURN_NONE;
  }
  if (status < 0) Py_RETURN_NONE;
  return PyLong_FromLong(status);
}

PyMethodDef methods[] = {
    {"call", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(call)), METH_FASTCALL, nullptr},
    {"layer", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer)), METH_FASTCALL, nullptr},
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
