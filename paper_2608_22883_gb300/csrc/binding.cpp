// The Python side of the drafter's cache (fovea_rotary_axes, fovea_cache_append,
// fovea_paged_attention, fovea_cache_keep, fovea_cache_fork): checks of the arguments,
// allocation of the outputs, the call.  The work of a decoding step is a few microseconds
// on the device; checked and allocated in Python, a call took 20 to 27 us of the host (a
// tensor's check 0.4, an allocation 1.6, forty arguments through ctypes 4), here it takes 5.5
// to 7.5 with one launch and 9.5 with two.
//
// Every function takes its arguments by place, as the wrappers in fovea.py give them (they
// have the documentation), works on the current stream of the current device, raises
// ValueError with the argument's name, and returns a status where the library has refused.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <optional>
#include <string>

#include "fovea.h"

namespace {

using at::ScalarType;
using at::Tensor;

struct Refused { std::string what; };

std::string sizes_of(at::IntArrayRef s) {
  std::string r = "[";
  for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + (s[i] < 0 ? std::string("any") : std::to_string(s[i]));
  return r + "]";
}

// A call's arguments and the device that it is made on.
struct Call {
  PyObject* const* args;
  mutable c10::DeviceIndex device = -1;      // the current one, asked once a tensor is on a GPU

  bool none(int i) const { return args[i] == Py_None; }
  const Tensor& tensor(int i, const char* name) const {
    if (!THPVariable_Check(args[i])) throw Refused{std::string(name) + " must be a CUDA tensor"};
    const Tensor& t = THPVariable_Unpack(args[i]);
    if (!t.is_cuda()) throw Refused{std::string(name) + " must be a CUDA tensor"};
    if (device < 0) device = c10::cuda::current_device();
    if (t.get_device() != device)
      throw Refused{std::string(name) + " is on cuda:" + std::to_string(t.get_device()) +
                    ", which is not the current device (cuda:" + std::to_string(device) + ")"};
    return t;
  }
  // A tensor of one of these types and of so many dims.
  const Tensor& typed(int i, const char* name, std::initializer_list<ScalarType> types, int64_t dims) const {
    const Tensor& t = tensor(i, name);
    bool ok = false;
    for (ScalarType type : types) ok = ok || t.scalar_type() == type;
    if (!ok) {
      std::string want;
      for (ScalarType type : types) want += (want.empty() ? "" : " or ") + std::string(c10::toString(type));
      throw Refused{std::string(name) + " has type " + c10::toString(t.scalar_type()) + "; expected " + want};
    }
    if (t.dim() != dims)
      throw Refused{std::string(name) + " has shape " + sizes_of(t.sizes()) + "; expected " + std::to_string(dims) +
                    " dims"};
    return t;
  }
  // A contiguous one of this shape (-1: any size).
  const Tensor& dense(int i, const char* name, ScalarType type, at::IntArrayRef shape) const {
    const Tensor& t = typed(i, name, {type}, (int64_t)shape.size());
    for (size_t d = 0; d < shape.size(); ++d)
      if (shape[d] >= 0 && t.size((int64_t)d) != shape[d])
        throw Refused{std::string(name) + " has shape " + sizes_of(t.sizes()) + "; expected " + sizes_of(shape)};
    if (!t.is_contiguous()) throw Refused{std::string(name) + " must be contiguous"};
    return t;
  }
  template <class T> T* maybe(int i, const char* name, ScalarType type, at::IntArrayRef shape) const {
    return none(i) ? nullptr : static_cast<T*>(dense(i, name, type, shape).data_ptr());
  }
  Tensor empty(at::IntArrayRef shape, ScalarType type) const {
    return at::detail::empty_cuda(shape, type, at::Device(at::kCUDA, device), std::nullopt);
  }
  void* stream() const { return c10::cuda::getCurrentCUDAStream(device).stream(); }
};

int dtype_of(ScalarType t) {
  return t == ScalarType::BFloat16 ? FOVEA_BF16 : t == ScalarType::Float ? FOVEA_FP32 : FOVEA_E4M3;
}
int int_of(int64_t n, const char* name) {
  if (n > INT32_MAX || n < INT32_MIN) throw Refused{std::string(name) + " is too large"};
  return (int)n;
}

// Rows [N, heads, dim] whose heads are contiguous.
struct Heads {
  const Tensor* t = nullptr;
  const void* at = nullptr;
  int n = 0, heads = 0, dim = 0;
  int64_t ld = 0, hs = 0;
  Heads() = default;
  Heads(const Call& c, int i, const char* name, std::initializer_list<ScalarType> types) {
    t = &c.typed(i, name, types, 3);
    if (t->stride(2) != 1 && t->size(2) > 1) throw Refused{std::string(name) + " must be contiguous along its heads"};
    at = t->data_ptr();
    n = int_of(t->size(0), name); heads = int_of(t->size(1), name); dim = int_of(t->size(2), name);
    ld = t->stride(0); hs = t->stride(1);
  }
  void same_rows(const char* name, const Heads& other) const {
    if (n != other.n || dim != other.dim)
      throw Refused{std::string(name) + " has shape " + sizes_of(t->sizes()) + "; the others are " +
                    sizes_of(other.t->sizes())};
  }
};

struct Rotary {
  const int32_t* positions = nullptr;
  int64_t ld = 0;
  int axes = 1, rot = 0;
  const double* frequencies = nullptr;
  const int32_t* axis = nullptr;
  Rotary() = default;
  Rotary(const Call& c, int i, int n) {      // positions, frequencies, axis
    const Tensor& p = c.typed(i, "positions", {ScalarType::Int}, 2);
    if (p.size(1) != n)
      throw Refused{"positions has shape " + sizes_of(p.sizes()) + "; expected " + std::to_string(n) + " columns"};
    if (p.stride(1) != 1 && n > 1) throw Refused{"positions must be contiguous along its rows"};
    positions = static_cast<const int32_t*>(p.data_ptr());
    axes = int_of(p.size(0), "positions");
    ld = axes > 1 ? p.stride(0) : n;
    const Tensor& f = c.dense(i + 1, "frequencies", ScalarType::Double, {-1});
    frequencies = static_cast<const double*>(f.data_ptr());
    rot = int_of(2 * f.size(0), "frequencies");
    axis = c.maybe<const int32_t>(i + 2, "axis", ScalarType::Int, {f.size(0)});
  }
};

struct Pages {
  void* k; void* v;
  int dtype, n_pages, heads, page, dim;
  const int32_t* table;
  int B, width;
  Pages(const Call& c, int i) {              // k_pages, v_pages, table
    const Tensor& kp = c.typed(i, "k_pages", {ScalarType::BFloat16, ScalarType::Float, ScalarType::Float8_e4m3fn}, 4);
    if (!kp.is_contiguous()) throw Refused{"k_pages must be contiguous"};
    k = kp.data_ptr();
    v = c.dense(i + 1, "v_pages", kp.scalar_type(), kp.sizes()).data_ptr();
    dtype = dtype_of(kp.scalar_type());
    n_pages = int_of(kp.size(0), "k_pages"); heads = int_of(kp.size(1), "k_pages");
    page = int_of(kp.size(2), "k_pages"); dim = int_of(kp.size(3), "k_pages");
    const Tensor& t = c.dense(i + 2, "table", ScalarType::Int, {-1, -1});
    table = static_cast<const int32_t*>(t.data_ptr());
    B = int_of(t.size(0), "table"); width = int_of(t.size(1), "table");
  }
  const float* scale(const Call& c, int i, const char* name) const {
    if (c.none(i)) return nullptr;
    if (dtype != FOVEA_E4M3) throw Refused{std::string(name) + " goes with a float8_e4m3fn cache, and only with it"};
    return c.maybe<const float>(i, name, ScalarType::Float, {heads});
  }
};

PyObject* status(fovea_status st) { return PyLong_FromLong(st); }
void put(PyObject* dict, const char* name, const Tensor& t) {
  PyObject* o = THPVariable_Wrap(t);
  if (o == nullptr || PyDict_SetItemString(dict, name, o) != 0) {
    Py_XDECREF(o);
    throw python_error();
  }
  Py_DECREF(o);
}

// The frame of every function: so many arguments, and exceptions turned into Python's.
template <class F>
PyObject* frame(PyObject* const* args, Py_ssize_t given, Py_ssize_t want, F body) {
  HANDLE_TH_ERRORS
  if (given != want) {
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, given);
    return nullptr;
  }
  try {
    return body(Call{args});
  } catch (const Refused& r) {
    PyErr_SetString(PyExc_ValueError, r.what.c_str());
    return nullptr;
  }
  END_HANDLE_TH_ERRORS
}

constexpr ScalarType kInt = ScalarType::Int;

// q, k, positions, frequencies, axis, adjacent, inverse
PyObject* rotary_axes(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return frame(args, given, 7, [&](const Call& c) -> PyObject* {
    const Heads q(c, 0, "q", {ScalarType::BFloat16, ScalarType::Float});
    const ScalarType type = q.t->scalar_type();
    Heads k;
    if (!c.none(1)) {
      k = Heads(c, 1, "k", {type});
      k.same_rows("k", q);
    }
    const Rotary r(c, 2, q.n);
    const Tensor q_out = c.empty({q.n, q.heads, q.dim}, type);
    Tensor k_out;
    if (k.t != nullptr) k_out = c.empty({k.n, k.heads, k.dim}, type);
    const fovea_status st = fovea_rotary_axes(
        q.at, q.ld, q.hs, q.heads, k.at, k.ld, k.hs, k.heads, q.n, q.dim, dtype_of(type), r.positions, r.ld, r.axes,
        r.frequencies, r.axis, r.rot, PyObject_IsTrue(args[5]), PyObject_IsTrue(args[6]), q_out.data_ptr(),
        k.t != nullptr ? k_out.data_ptr() : nullptr, c.stream());
    if (st != FOVEA_OK) return status(st);
    PyObject* pair = PyTuple_New(2);
    if (pair == nullptr) throw python_error();
    PyTuple_SET_ITEM(pair, 0, THPVariable_Wrap(q_out));
    PyTuple_SET_ITEM(pair, 1, k.t != nullptr ? THPVariable_Wrap(k_out) : Py_NewRef(Py_None));
    return pair;
  });
}

// k, v, k_pages, v_pages, table, sequence, entry, k_scale, v_scale, q, positions, frequencies, axis, adjacent
PyObject* cache_append(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return frame(args, given, 14, [&](const Call& c) -> PyObject* {
    const Heads k(c, 0, "k", {ScalarType::BFloat16, ScalarType::Float});
    const ScalarType type = k.t->scalar_type();
    const Heads v(c, 1, "v", {type});
    v.same_rows("v", k);
    const Pages p(c, 2);
    if (v.heads != k.heads || p.heads != k.heads || p.dim != k.dim)
      throw Refused{"k " + sizes_of(k.t->sizes()) + ", v " + sizes_of(v.t->sizes()) + " and pages of " +
                    std::to_string(p.heads) + " heads of " + std::to_string(p.dim) + " differ in size"};
    const auto* sequence = static_cast<const int32_t*>(c.dense(5, "sequence", kInt, {k.n}).data_ptr());
    const auto* entry = static_cast<const int32_t*>(c.dense(6, "entry", kInt, {k.n}).data_ptr());
    const float* k_scale = p.scale(c, 7, "k_scale");
    const float* v_scale = p.scale(c, 8, "v_scale");
    if (c.none(10) != c.none(11)) throw Refused{"positions and frequencies go together"};
    if (c.none(10) && !(c.none(9) && c.none(12))) throw Refused{"q and axis go with positions and frequencies"};
    Rotary r;
    if (!c.none(10)) r = Rotary(c, 10, k.n);
    Heads q;
    Tensor out;
    if (!c.none(9)) {
      q = Heads(c, 9, "q", {type});
      q.same_rows("q", k);
      out = c.empty({q.n, q.heads, q.dim}, type);
    }
    const fovea_status st = fovea_cache_append(
        q.at, q.ld, q.hs, q.heads, k.at, k.ld, k.hs, v.at, v.ld, v.hs, k.n, dtype_of(type), r.positions, r.ld, r.axes,
        r.frequencies, r.axis, r.rot, PyObject_IsTrue(args[13]), q.t != nullptr ? out.data_ptr() : nullptr, p.k, p.v,
        p.dtype, k_scale, v_scale, p.n_pages, p.page, p.heads, p.dim, p.table, p.B, p.width, sequence, entry,
        c.stream());
    if (st != FOVEA_OK) return status(st);
    return q.t != nullptr ? THPVariable_Wrap(out) : Py_NewRef(Py_None);
  });
}

// q, k_pages, v_pages, table, lens, tree, scale, k_scale, v_scale, want_lse, workspace
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return frame(args, given, 11, [&](const Call& c) -> PyObject* {
    const Heads q(c, 0, "q", {ScalarType::BFloat16, ScalarType::Float});
    const ScalarType type = q.t->scalar_type();
    const Pages p(c, 1);
    if ((type == ScalarType::Float) != (p.dtype == FOVEA_FP32))
      throw Refused{"fp32 rows go with an fp32 cache, bf16 rows with a bf16 or float8_e4m3fn one"};
    if (p.dim != q.dim || p.heads == 0 || q.heads % p.heads != 0)
      throw Refused{"q " + sizes_of(q.t->sizes()) + " does not go with pages of " + std::to_string(p.heads) +
                    " heads of " + std::to_string(p.dim)};
    if (p.B == 0 ? q.n != 0 : q.n % p.B != 0)
      throw Refused{"q has " + std::to_string(q.n) + " rows, which are not the same number for each of " +
                    std::to_string(p.B) + " sequences"};
    const int nodes = p.B == 0 ? 1 : q.n / p.B;
    const int32_t* lens = static_cast<const int32_t*>(c.dense(4, "lens", kInt, {p.B}).data_ptr());
    const int32_t* tree = nullptr;
    int trees = 0;
    if (!c.none(5)) {
      const Tensor& t = c.dense(5, "tree", kInt, {-1, nodes, (nodes + 31) / 32});
      if (t.size(0) != 1 && t.size(0) != p.B)
        throw Refused{"tree has " + std::to_string(t.size(0)) + " trees; expected " + std::to_string(p.B) + " or 1"};
      trees = (int)t.size(0);
      tree = static_cast<const int32_t*>(t.data_ptr());
    }
    const float* k_scale = p.scale(c, 7, "k_scale");
    const float* v_scale = p.scale(c, 8, "v_scale");
    double scale = 1.0 / std::sqrt((double)q.dim);
    if (!c.none(6)) {
      scale = PyFloat_AsDouble(args[6]);
      if (scale == -1.0 && PyErr_Occurred()) throw python_error();
    }
    Tensor out = c.empty({q.n, q.heads, q.dim}, type), lse, scratch;
    const bool want_lse = PyObject_IsTrue(args[9]);
    if (want_lse) lse = c.empty({q.n, q.heads}, ScalarType::Float);
    if (q.n > 0) {
      size_t bytes = 0;
      void* workspace = nullptr;
      if (!c.none(10)) {
        const Tensor& w = c.dense(10, "workspace", ScalarType::Byte, {-1});
        workspace = w.data_ptr();
        bytes = (size_t)w.numel();
      } else {
        const fovea_status st = fovea_paged_attention_workspace_size(p.B, nodes, q.heads, p.heads, q.dim, p.dtype, &bytes);
        if (st != FOVEA_OK) return status(st);
        scratch = c.empty({(int64_t)bytes}, ScalarType::Byte);
        workspace = scratch.data_ptr();
      }
      const fovea_status st = fovea_paged_attention(
          q.at, q.ld, q.hs, q.heads, p.k, p.v, p.dtype, k_scale, v_scale, p.n_pages, p.page, p.heads, p.dim, p.table,
          p.B, p.width, lens, nodes, tree, trees, (float)scale, out.data_ptr(),
          want_lse ? static_cast<float*>(lse.data_ptr()) : nullptr, workspace, bytes, c.stream());
      if (st != FOVEA_OK) return status(st);
    }
    PyObject* r = PyDict_New();
    if (r == nullptr) throw python_error();
    put(r, "out", out);
    if (want_lse) put(r, "lse", lse);
    return r;
  });
}

// k_pages, v_pages, table, lens, nodes, size
PyObject* cache_keep(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return frame(args, given, 6, [&](const Call& c) -> PyObject* {
    const Pages p(c, 0);
    const auto* lens = static_cast<const int32_t*>(c.dense(3, "lens", kInt, {p.B}).data_ptr());
    const Tensor& nodes = c.dense(4, "nodes", kInt, {p.B, -1});
    const long size = PyLong_AsLong(args[5]);
    if (size == -1 && PyErr_Occurred()) throw python_error();
    const Tensor out = c.empty({p.B}, kInt);
    const fovea_status st = fovea_cache_keep(
        p.k, p.v, p.dtype, p.n_pages, p.page, p.heads, p.dim, p.table, p.B, p.width, lens,
        static_cast<const int32_t*>(nodes.data_ptr()), int_of(nodes.size(1), "nodes"), int_of(size, "size"),
        static_cast<int32_t*>(out.data_ptr()), c.stream());
    return st != FOVEA_OK ? status(st) : THPVariable_Wrap(out);
  });
}

// k_pages, v_pages, table, lens, parents, keep, room, width
PyObject* cache_fork(PyObject*, PyObject* const* args, Py_ssize_t given) {
  return frame(args, given, 8, [&](const Call& c) -> PyObject* {
    const Pages p(c, 0);
    const auto* lens = static_cast<const int32_t*>(c.dense(3, "lens", kInt, {p.B}).data_ptr());
    const Tensor& parents = c.dense(4, "parents", kInt, {-1});
    const int C = int_of(parents.size(0), "parents");
    const auto* keep = c.maybe<const int32_t>(5, "keep", kInt, {C});
    const auto* room = c.maybe<const int32_t>(6, "room", kInt, {C});
    long width = p.width;
    if (!c.none(7)) {
      width = PyLong_AsLong(args[7]);
      if (width == -1 && PyErr_Occurred()) throw python_error();
    }
    if (width < 1) throw Refused{"width " + std::to_string(width) + " is below 1"};
    const Tensor table = c.empty({C, int_of(width, "width")}, kInt), new_lens = c.empty({C}, kInt),
                 left = c.empty({1}, kInt);
    const fovea_status st = fovea_cache_fork(
        p.k, p.v, p.dtype, p.n_pages, p.page, p.heads, p.dim, p.table, p.B, p.width, lens,
        static_cast<const int32_t*>(parents.data_ptr()), keep, room, C, static_cast<int32_t*>(table.data_ptr()),
        (int)width, static_cast<int32_t*>(new_lens.data_ptr()), static_cast<int32_t*>(left.data_ptr()), c.stream());
    if (st != FOVEA_OK) return status(st);
    PyObject* r = PyDict_New();
    if (r == nullptr) throw python_error();
    put(r, "table", table);
    put(r, "lens", new_lens);
    put(r, "free", left);
    return r;
  });
}

#define FOVEA_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef kMethods[] = {FOVEA_METHOD(rotary_axes), FOVEA_METHOD(cache_append), FOVEA_METHOD(paged_attention),
                          FOVEA_METHOD(cache_keep), FOVEA_METHOD(cache_fork), {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "fovea_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_fovea_binding() { return PyModule_Create(&kModule); }
