// Native marshalling of torch tensors into the C ABI for the calls that a
// program makes once a layer and token (Python module _marshal).
//
// Types, devices, shapes and strides are read from the tensors directly: the
// same checks in Python took 2 to 5 us of a call, where launching takes 3
// (appending 9 tokens 9.5 us -> 5.5, a tree's masks 5.9 -> 3.6).  binding.py holds
// the functions that users call, their defaults and documentation.
//
// A function takes the addresses of its structs (dllm_kv_pages, dllm_rotary) and
// the device they belong to, then tensors or None; it raises ValueError for
// tensors that do not fit one another and returns the status of the C entry.
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>

#include <algorithm>
#include <cmath>
#include <exception>

#include "dllm_rps.h"

namespace {

// a Python error that has been set
struct Raised {};
[[noreturn]] void refuse(const char* text) {
  PyErr_SetString(PyExc_ValueError, text);
  throw Raised{};
}

int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}
int32_t number(PyObject* o) {
  const int64_t v = whole(o);
  if (v < INT32_MIN || v > INT32_MAX) {
    PyErr_SetString(PyExc_OverflowError, "a number of more than 32 bits");
    throw Raised{};
  }
  return int32_t(v);
}
template <typename T>
const T* struct_at(PyObject* o) {
  return reinterpret_cast<const T*>(intptr_t(whole(o)));
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "a torch tensor is needed, not %s", Py_TYPE(o)->tp_name);
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}

// the device of a call, which has to be the current one, and its stream
struct Place {
  int index;
  explicit Place(PyObject* o) : index(number(o)) {}
  dllm_stream stream(PyObject* o) const {
    if (int(c10::hip::current_device()) != index) refuse("the arrays are on another device than the current one");
    if (o != Py_None) return reinterpret_cast<dllm_stream>(intptr_t(whole(o)));
    return c10::hip::getCurrentHIPStream(c10::DeviceIndex(index)).stream();
  }
};

// a contiguous int32 tensor of the given sizes (n entries, or n x rows [x words]); None is NULL
int32_t* ints(const Place& p, PyObject* o, const char* text, int64_t n, int64_t rows = -1, int64_t words = -1) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  const bool fits = rows < 0 ? t.numel() == n
                             : t.dim() == (words < 0 ? 2 : 3) && t.size(0) == n && t.size(1) == rows &&
                                   (words < 0 || t.size(2) == words);
  if (!fits || t.scalar_type() != at::kInt || t.get_device() != p.index || !t.is_contiguous()) refuse(text);
  return static_cast<int32_t*>(t.data_ptr());
}
constexpr const char* kLists =
    "sequence lists, counts and status are contiguous int32 tensors, one value an entry, beside the other arrays";
constexpr const char* kGrids =
    "positions, parents and paths are contiguous int32 tensors [entries, rows], beside the other arrays";
constexpr const char* kMasks = "a mask is a contiguous int32 tensor [entries, rows, words of 32 rows] beside the pages";

struct Scratch {
  void* p;
  size_t bytes;
};
Scratch scratch(const Place& p, PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.get_device() != p.index || !t.is_contiguous()) refuse("the workspace must be contiguous and beside the pages");
  return Scratch{t.data_ptr(), t.nbytes()};
}

// [entries, rows, heads, head_dim] of any strides over contiguous head_dim
struct Sizes {
  int64_t n, rows, heads;
};
Sizes sizes(PyObject* o, int64_t hd) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 4 || t.size(3) != hd) refuse("rows are tensors [entries, rows, heads, head_dim] of the head_dim given");
  if (t.size(2) > INT32_MAX) refuse("too many heads");
  return Sizes{t.size(0), t.size(1), t.size(2)};
}
dllm_rows rows(const Place& p, PyObject* o, const Sizes& s, int64_t hd, at::ScalarType type) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 4 || t.size(0) != s.n || t.size(1) != s.rows || t.size(2) != s.heads || t.size(3) != hd)
    refuse("rows of one call need the same entries, rows and head_dim, and an output those of its input");
  if (t.stride(3) != 1 || t.scalar_type() != type || t.get_device() != p.index)
    refuse("rows must be contiguous, of one type, and on the device of the other arrays");
  // a dimension of one has no stride to speak of
  return dllm_rows{t.data_ptr(), s.n > 1 ? t.stride(0) : 0, s.rows > 1 ? t.stride(1) : 0, s.heads > 1 ? t.stride(2) : 0};
}
int32_t count(int64_t v) {
  if (v > INT32_MAX) refuse("too many rows or entries");
  return int32_t(v);
}
at::ScalarType type_of(const dllm_kv_pages* p) { return p->dtype == DLLM_BF16 ? at::kBFloat16 : at::kFloat; }

template <typename F>
PyObject* guarded(F&& f) {
  try {
    return PyLong_FromLong(long(f()));
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}
template <typename F>
dllm_status unlocked(F&& f) {
  dllm_status st;
  Py_BEGIN_ALLOW_THREADS st = f();
  Py_END_ALLOW_THREADS return st;
}
void arguments(Py_ssize_t got, Py_ssize_t want) {
  if (got == want) return;
  PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", want, got);
  throw Raised{};
}

// rot, device, q, q_out, k, k_out, pos, pos_offset, n_rows, stream
PyObject* rotary_rows_(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    arguments(n_args, 10);
    const auto* rot = struct_at<dllm_rotary>(a[0]);
    const Place p(a[1]);
    const bool has_q = a[2] != Py_None, has_k = a[4] != Py_None;
    if (!has_q && !has_k) refuse("neither queries nor keys");
    const at::ScalarType type = tensor(has_q ? a[2] : a[4]).scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) refuse("rows are bf16 or fp32");
    const int64_t hd = rot->head_dim;
    const Sizes first = sizes(has_q ? a[2] : a[4], hd);
    dllm_rows q{}, qo{}, k{}, ko{};
    Sizes sq{first.n, first.rows, 0}, sk = sq;
    if (has_q) {
      sq.heads = first.heads;
      q = rows(p, a[2], sq, hd, type);
      qo = rows(p, a[3], sq, hd, type);
    }
    if (has_k) {
      sk.heads = sizes(a[4], hd).heads;
      k = rows(p, a[4], sk, hd, type);
      ko = rows(p, a[5], sk, hd, type);
    }
    const int32_t* pos = ints(p, a[6], kGrids, first.n, first.rows);
    const int32_t offset = number(a[7]), n = count(first.n), max_rows = count(first.rows);
    const int32_t* n_rows = ints(p, a[8], kLists, n);
    const dllm_stream s = p.stream(a[9]);
    return unlocked([&] {
      return rotary_rows(rot, type == at::kBFloat16 ? DLLM_BF16 : DLLM_F32, pos, offset, n, max_rows, n_rows,
                         int32_t(sq.heads), &q, &qo, int32_t(sk.heads), &k, &ko, s);
    });
  });
}

// pages, device, layer, seqs, n_rows, rot, rot's device, pos, q, q_out, k, v, stream
PyObject* kv_pages_append_(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    arguments(n_args, 13);
    const auto* pages = struct_at<dllm_kv_pages>(a[0]);
    const Place p(a[1]);
    const int32_t layer = number(a[2]);
    const auto* rot = struct_at<dllm_rotary>(a[5]);
    if (number(a[6]) != p.index) refuse("the rotation is on another device than the pages");
    const at::ScalarType type = type_of(pages);
    const int64_t hd = pages->head_dim;
    Sizes s = sizes(a[10], hd);
    if (s.heads != pages->n_kv_heads) refuse("k and v need the pages' heads and head_dim and the same shape");
    const dllm_rows k = rows(p, a[10], s, hd, type), v = rows(p, a[11], s, hd, type);
    dllm_rows q{}, qo{};
    int64_t heads = 0;
    if (a[8] != Py_None) {
      s.heads = heads = sizes(a[8], hd).heads;
      q = rows(p, a[8], s, hd, type);
      qo = rows(p, a[9], s, hd, type);
    }
    const int32_t n = count(s.n), max_rows = count(s.rows);
    const int32_t *seqs = ints(p, a[3], kLists, n), *n_rows = ints(p, a[4], kLists, n), *pos = ints(p, a[7], kGrids, n, max_rows);
    const dllm_stream st = p.stream(a[12]);
    return unlocked([&] {
      return kv_pages_append(pages, layer, seqs, n, max_rows, n_rows, rot, pos, int32_t(heads), &q, &qo, &k, &v, st);
    });
  });
}

// pages, device, seqs, n_rows, parent, mask, pos, stream
PyObject* kv_pages_tree_(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    arguments(n_args, 8);
    const auto* pages = struct_at<dllm_kv_pages>(a[0]);
    const Place p(a[1]);
    const at::Tensor& t = tensor(a[4]);
    if (t.dim() != 2) refuse(kGrids);
    const int32_t n = count(t.size(0)), max_rows = count(t.size(1));
    const int32_t *seqs = ints(p, a[2], kLists, n), *n_rows = ints(p, a[3], kLists, n);
    const int32_t* parent = ints(p, a[4], kGrids, n, max_rows);
    int32_t *mask = ints(p, a[5], kMasks, n, max_rows, (int64_t(max_rows) + 31) / 32), *pos = ints(p, a[6], kGrids, n, max_rows);
    const dllm_stream s = p.stream(a[7]);
    return unlocked([&] {
      return kv_pages_tree(pages, seqs, n, max_rows, n_rows, parent, reinterpret_cast<uint32_t*>(mask), pos, s);
    });
  });
}

// pages, device, layer, seqs, n_rows, q, out, mask, prefix_seq, shared_len, max_len or None, scale or None, ws, stream
PyObject* kv_pages_attention_tree_(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    arguments(n_args, 14);
    const auto* pages = struct_at<dllm_kv_pages>(a[0]);
    const Place p(a[1]);
    const int64_t hd = pages->head_dim;
    const Sizes s = sizes(a[5], hd);
    const dllm_rows q = rows(p, a[5], s, hd, type_of(pages)), out = rows(p, a[6], s, hd, type_of(pages));
    const int32_t n = count(s.n), max_rows = count(s.rows), heads = count(s.heads);
    const int32_t layer = number(a[2]), *seqs = ints(p, a[3], kLists, n), *n_rows = ints(p, a[4], kLists, n);
    const int32_t* mask = ints(p, a[7], kMasks, n, max_rows, (int64_t(max_rows) + 31) / 32);
    const int32_t prefix = number(a[8]), shared = number(a[9]);
    const int32_t most = a[10] == Py_None ? int32_t(std::min<int64_t>(int64_t(pages->max_blocks) * pages->page_len, INT32_MAX))
                                           : number(a[10]);
    double scale = 1.0 / std::sqrt(double(hd));
    if (a[11] != Py_None) {
      scale = PyFloat_AsDouble(a[11]);
      if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
    }
    const Scratch ws = scratch(p, a[12]);
    const dllm_stream st = p.stream(a[13]);
    return unlocked([&] {
      return kv_pages_attention_tree(pages, layer, seqs, n, max_rows, n_rows, heads, &q, &out,
                                     reinterpret_cast<const uint32_t*>(mask), prefix, shared, most, float(scale), ws.p,
                                     ws.bytes, st);
    });
  });
}

// pages, device, seqs, rows, n_rows, path, n_path, status, ws, stream
PyObject* kv_pages_accept_(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
  return guarded([&] {
    arguments(n_args, 10);
    const auto* pages = struct_at<dllm_kv_pages>(a[0]);
    const Place p(a[1]);
    const at::Tensor& t = tensor(a[5]);
    if (t.dim() != 2) refuse(kGrids);
    const int32_t n = count(t.size(0)), max_path = count(t.size(1)), max_rows = number(a[3]);
    const int32_t *seqs = ints(p, a[2], kLists, n), *n_rows = ints(p, a[4], kLists, n);
    const int32_t *path = ints(p, a[5], kGrids, n, max_path), *n_path = ints(p, a[6], kLists, n);
    int32_t* status = ints(p, a[7], kLists, 1);
    const Scratch ws = scratch(p, a[8]);
    const dllm_stream s = p.stream(a[9]);
    return unlocked([&] {
      return kv_pages_accept(pages, seqs, n, max_rows, n_rows, path, max_path, n_path, status, ws.p, ws.bytes, s);
    });
  });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
constexpr PyMethodDef method(const char* name) {
  return PyMethodDef{name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}
PyMethodDef kMethods[] = {method<rotary_rows_>("rotary_rows"),
                          method<kv_pages_append_>("kv_pages_append"),
                          method<kv_pages_tree_>("kv_pages_tree"),
                          method<kv_pages_attention_tree_>("kv_pages_attention_tree"),
                          method<kv_pages_accept_>("kv_pages_accept"),
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&kModule); }
