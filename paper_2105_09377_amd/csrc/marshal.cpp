// Native half of the Python binding: torch tensors -> `gs_ap` descriptors -> C entry point.
//
// A call through ctypes cost 8 us on the host for a product and 10 for a convolution, of which the
// entry point itself (checks and one launch) is 3: for small problems the descriptors, built
// field by field in Python, were what a pass waited for.  Here a call reads the tensors directly.
// No arithmetic, no fallback; the entry points are those that binding.py has loaded (`bind`).
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <utility>
#include <vector>

#include "../../include/glenside.h"

namespace {

struct Failed {};   // a Python error is set

struct Api {
  decltype(&glenside_windows_out_shape) windows_out_shape;
  decltype(&glenside_access_windows) access_windows;
  decltype(&glenside_cartesian_dot) cartesian_dot;
  decltype(&glenside_conv2d_direct) conv2d_direct, conv2d_im2col, conv2d_direct_packed;
  decltype(&glenside_conv2d_direct_packed_with_projection) conv2d_direct_packed_with_projection;
  decltype(&glenside_conv2d_direct_workspace) conv2d_direct_workspace, conv2d_im2col_workspace;
  decltype(&glenside_reduce) reduce;
  decltype(&glenside_windows_reduce) windows_reduce;
  decltype(&glenside_pair_reduce) pair_reduce;
  decltype(&glenside_depthwise_conv2d) depthwise_conv2d;
  decltype(&glenside_transpose) transpose;
  decltype(&glenside_program_shape) program_shape;
  decltype(&glenside_program_workspace) program_workspace;
  decltype(&glenside_program_eval) program_eval;
  decltype(&glenside_mx4_sizes) mx4_sizes;
  decltype(&glenside_mx4_quantize) mx4_quantize;
  decltype(&glenside_mx4_dequantize) mx4_dequantize;
  decltype(&glenside_mx4_dot) mx4_dot;
  decltype(&glenside_mx4_dot_workspace) mx4_dot_workspace;
  decltype(&glenside_mx4_weight_dot) mx4_weight_dot;
  decltype(&glenside_mx4_weight_dot_workspace) mx4_weight_dot_workspace;
  decltype(&glenside_mx4_cache_bytes) mx4_cache_bytes;
  decltype(&glenside_mx4_cache_append) mx4_cache_append;
  decltype(&glenside_mx4_cache_read) mx4_cache_read;
  decltype(&glenside_mx4_attend) mx4_attend;
  decltype(&glenside_mx4_attend_workspace) mx4_attend_workspace;
  decltype(&glenside_f8_sizes) f8_sizes;
  decltype(&glenside_f8_quantize) f8_quantize;
  decltype(&glenside_f8_dequantize) f8_dequantize;
  decltype(&glenside_norm) norm;
  decltype(&glenside_f8_norm) f8_norm;
  decltype(&glenside_f8_dot) f8_dot;
  decltype(&glenside_f8_dot_workspace) f8_dot_workspace;
  decltype(&glenside_f8_expert_dot) f8_expert_dot;
  decltype(&glenside_f8_expert_dot_workspace) f8_expert_dot_workspace;
  decltype(&glenside_expert_sort) expert_sort;
  decltype(&glenside_expert_sort_workspace) expert_sort_workspace;
  decltype(&glenside_expert_split) expert_split;
  decltype(&glenside_expert_join) expert_join;
  decltype(&glenside_expert_join_grad) expert_join_grad;
} api;
PyObject* error_class;

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_AttributeError, "'%.100s' object is no tensor", Py_TYPE(o)->tp_name);
    throw Failed{};
  }
  return THPVariable_Unpack(o);
}

int dtype_code(at::ScalarType t) {
  switch (t) {
    case at::kChar: return GS_I8;
    case at::kInt: return GS_I32;
    case at::kBFloat16: return GS_BF16;
    case at::kFloat: return GS_F32;
    case at::kFloat8_e4m3fn: return GS_F8;
    default: PyErr_SetString(PyExc_KeyError, c10::toString(t)); throw Failed{};
  }
}

// Descriptor of a contiguous tensor with n_access access dimensions (the library refuses impossible ones).
gs_ap describe(const at::Tensor& t, int64_t n_access) {
  gs_ap a{};
  if (!t.is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "access patterns are dense row-major tensors");
    throw Failed{};
  }
  const auto sizes = t.sizes();
  if (sizes.size() > GS_MAX_RANK) {
    PyErr_SetString(PyExc_ValueError, "rank above GS_MAX_RANK");
    throw Failed{};
  }
  a.data = t.data_ptr();
  a.dtype = dtype_code(t.scalar_type());
  a.rank = int32_t(sizes.size());
  a.n_access = int32_t(n_access);
  for (size_t i = 0; i < sizes.size(); ++i) a.shape[i] = sizes[i];
  return a;
}
// Every dimension an access dimension: results and element-wise operands.
gs_ap describe_all(const at::Tensor& t) { return describe(t, t.dim()); }

int64_t integer(PyObject* o) {
  if (PyLong_CheckExact(o)) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
  }
  PyObject* l = PyNumber_Long(o);
  if (!l) throw Failed{};
  const int64_t v = PyLong_AsLongLong(l);
  Py_DECREF(l);
  if (v == -1 && PyErr_Occurred()) throw Failed{};
  return v;
}

// An operator or activation code: integers only, a float is no code.
int code(PyObject* o) {
  PyObject* l = PyNumber_Index(o);
  if (!l) throw Failed{};
  const int v = int(PyLong_AsUnsignedLongMask(l));
  Py_DECREF(l);
  return v;
}

// A new reference, held until the end of the scope.
struct Owned {
  PyObject* object;
  explicit Owned(PyObject* o) : object(o) {
    if (!o) throw Failed{};
  }
  ~Owned() { Py_DECREF(object); }
  Owned(const Owned&) = delete;
};

// The items of a mapping, held until the end of the scope: all of them are taken before any is converted, which
// may run any code.  Twice cheaper than a copy of the dict, which only other mappings need.
struct Items {
  std::vector<std::pair<PyObject*, PyObject*>> items;
  explicit Items(PyObject* mapping) {
    if (PyDict_CheckExact(mapping)) {
      take(mapping);
      return;
    }
    const Owned copy(PyDict_New());
    if (PyDict_Update(copy.object, mapping)) throw Failed{};
    take(copy.object);
  }
  ~Items() {
    for (const auto& i : items) {
      Py_DECREF(i.first);
      Py_DECREF(i.second);
    }
  }
  Items(const Items&) = delete;

 private:
  void take(PyObject* dict) {
    items.reserve(size_t(PyDict_GET_SIZE(dict)));
    PyObject *key, *value;
    for (Py_ssize_t pos = 0; PyDict_Next(dict, &pos, &key, &value);) {
      Py_INCREF(key);
      Py_INCREF(value);
      items.push_back({key, value});
    }
  }
};

// A sequence of integers; None = absent (a null pointer at the C boundary).
struct Ints {
  int64_t v[2 * GS_MAX_RANK] = {};
  int n = 0;
  bool present = false;
  explicit Ints(PyObject* o) {
    if (o == Py_None) return;
    present = true;
    // sized, as a generator is not; a tuple of its own, for the conversions may run any code
    if (PyObject_Size(o) < 0) throw Failed{};
    const Owned seq(PySequence_Tuple(o));
    const Py_ssize_t len = PyTuple_GET_SIZE(seq.object);
    if (len > 2 * GS_MAX_RANK) {
      PyErr_SetString(PyExc_ValueError, "too many integers");
      throw Failed{};
    }
    for (Py_ssize_t i = 0; i < len; ++i) v[i] = integer(PyTuple_GET_ITEM(seq.object, i));
    n = int(len);
  }
  const int64_t* get() const { return present ? v : nullptr; }
};

void* stream_of(const at::Tensor& t) {
  return t.is_cuda() ? static_cast<void*>(c10::hip::getCurrentHIPStream(t.get_device()).stream()) : nullptr;
}

[[noreturn]] void refuse(int status, const char* where) {
  PyObject* args = Py_BuildValue("(is)", status, where);
  if (args) {
    PyErr_SetObject(error_class, args);
    Py_DECREF(args);
  }
  throw Failed{};
}

// The interpreter lock released until the end of the scope, also where that is left by an exception.
struct Unlocked {
  PyThreadState* const state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};

// Runs an entry point without the interpreter lock; a status other than GS_OK becomes GlensideError.
template <typename F>
void call(const char* where, F&& f) {
  int status;
  {
    const Unlocked unlocked;
    status = f();
  }
  if (status != GS_OK) refuse(status, where);
}

// The result: `out` as given, or a new tensor of this shape, of `dtype` (a torch dtype, None = `otherwise`).
struct Result {
  PyObject* object;      // a new reference
  at::Tensor value;
  // cleared: a new tensor is zeros, of which a call writes a part.
  Result(PyObject* out, PyObject* dtype, at::ScalarType otherwise, const int64_t* shape, int rank, const at::Tensor& like, bool cleared = false) {
    if (out != Py_None) {
      value = tensor(out);
      object = out;
      Py_INCREF(out);
      return;
    }
    at::ScalarType st = otherwise;
    if (dtype != Py_None) {
      if (!THPDtype_Check(dtype)) {
        PyErr_SetString(PyExc_TypeError, "out_dtype is a torch dtype");
        throw Failed{};
      }
      st = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
    }
    value = at::empty(at::IntArrayRef(shape, rank), at::TensorOptions().dtype(st).device(like.device()));
    if (cleared) value.zero_();
    object = THPVariable_Wrap(value);
    if (!object) throw Failed{};
  }
};

template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t want, F&& f) {
  if (got != want) {
    PyErr_Format(PyExc_TypeError, "%zd arguments are wanted", want);
    return nullptr;
  }
  PyObject* r = nullptr;       // set as soon as there is a result, so that a failed call releases it
  try {
    f(r);
    return r;
  } catch (const Failed&) {
  } catch (...) {       // torch's own classes: torch.OutOfMemoryError stays what it is
    torch::translate_exception_to_python(std::current_exception());
  }
  Py_XDECREF(r);
  return nullptr;
}

at::ScalarType sum_type(const at::Tensor& x) { return x.scalar_type() == at::kChar ? at::kInt : at::kFloat; }

// cartesian_dot(a0, a1, n_access0, n_access1, out_dtype, act, out)
PyObject* py_cartesian_dot(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 7, [&](PyObject*& r) {
    const at::Tensor &a0 = tensor(p[0]), &a1 = tensor(p[1]);
    const int64_t n0 = integer(p[2]), n1 = integer(p[3]);
    const int act = code(p[5]);
    int64_t shape[2 * GS_MAX_RANK];
    int rank = 0;
    if (p[6] == Py_None) {
      for (int64_t i = 0; i < n0 && i < a0.dim() && i < GS_MAX_RANK; ++i) shape[rank++] = a0.size(i);
      for (int64_t i = 0; i < n1 && i < a1.dim() && i < GS_MAX_RANK; ++i) shape[rank++] = a1.size(i);
    }
    Result out(p[6], p[4], sum_type(a0), shape, rank, a0);
    r = out.object;
    gs_ap x = describe(a0, n0), y = describe(a1, n1), o = describe_all(out.value);
    void* s = stream_of(a0);
    call("cartesian_dot", [&] { return api.cartesian_dot(&x, &y, &o, act, nullptr, 0, s); });
  });
}

// conv(form, x, w, stride, pad, residual, act, out_dtype, out, workspace); form 0 direct, 1 packed, 2 im2col
PyObject* py_conv(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 10, [&](PyObject*& r) {
    const int64_t form = integer(p[0]);
    const at::Tensor &x = tensor(p[1]), &w = tensor(p[2]);
    const Ints stride(p[3]), pad(p[4]);
    const int act = code(p[6]);
    gs_ap xa = describe(x, 1), wa = describe(w, 1);
    int64_t shape[4] = {0, 0, 0, 0};
    if (p[8] == Py_None) {
      // H', W' from the shape rule of `windows` (window (C,Kh,Kw), strides (1,Sh,Sw))
      if (x.dim() < 2 || w.dim() != 4 || stride.n < 2 || pad.n < 2) {
        PyErr_SetString(PyExc_IndexError, "activations (N,C,H,W), weights (O,C,Kh,Kw), two strides and pads are wanted");
        throw Failed{};
      }
      const int64_t window[3] = {x.size(1), w.size(2), w.size(3)}, st[3] = {1, stride.v[0], stride.v[1]}, pd[3] = {0, pad.v[0], pad.v[1]};
      gs_ap want{};
      if (x.dim() != 4) {
        PyErr_SetString(PyExc_IndexError, "activations (N,C,H,W) are wanted");
        throw Failed{};
      }
      call("windows_out_shape", [&] { return api.windows_out_shape(&xa, window, st, pd, pd, &want); });
      shape[0] = x.size(0);
      shape[1] = w.size(0);
      shape[2] = want.shape[2];
      shape[3] = want.shape[3];
    }
    Result out(p[8], p[7], sum_type(x), shape, 4, x);
    r = out.object;
    at::Tensor ws;
    if (p[9] != Py_None) {
      ws = tensor(p[9]);
    } else {
      const size_t need = form == 2 ? api.conv2d_im2col_workspace(&xa, &wa, stride.get(), pad.get())
                                    : api.conv2d_direct_workspace(&xa, &wa, stride.get(), pad.get());
      ws = at::empty({int64_t(need > 16 ? need : 16)}, at::TensorOptions().dtype(at::kByte).device(x.device()));
    }
    gs_ap oa = describe(out.value, 4), ra{};
    if (p[5] != Py_None) ra = describe_all(tensor(p[5]));
    const gs_ap* res = p[5] != Py_None ? &ra : nullptr;
    void *wsp = ws.data_ptr(), *s = stream_of(x);
    const size_t bytes = size_t(ws.numel());
    const auto fn = form == 0 ? api.conv2d_direct : form == 1 ? api.conv2d_direct_packed : api.conv2d_im2col;
    call(form == 0 ? "glenside_conv2d_direct" : form == 1 ? "glenside_conv2d_direct_packed" : "glenside_conv2d_im2col",
         [&] { return fn(&xa, &wa, stride.get(), pad.get(), res, act, &oa, wsp, bytes, s); });
  });
}

// conv_with_projection(x, w, packed, w_proj, packed_proj, stride, pad, act, out, out_proj)
PyObject* py_conv_with_projection(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 10, [&](PyObject*& r) {
    const at::Tensor &x = tensor(p[0]), &packed = tensor(p[2]), &packed_proj = tensor(p[4]);
    const Ints stride(p[5]), pad(p[6]);
    const int act = code(p[7]);
    const gs_ap xa = describe(x, 1), wa = describe(tensor(p[1]), 1), pa = describe(tensor(p[3]), 1);
    gs_ap oa = describe(tensor(p[8]), 4), qa = describe(tensor(p[9]), 4);
    void* s = stream_of(x);
    call("glenside_conv2d_direct_packed_with_projection", [&] {
      return api.conv2d_direct_packed_with_projection(&xa, &wa, stride.get(), pad.get(), act, &oa, packed.data_ptr(), size_t(packed.numel()),
                                                      &pa, &qa, packed_proj.data_ptr(), size_t(packed_proj.numel()), s);
    });
    Py_INCREF(p[8]);
    r = p[8];
  });
}

at::ScalarType reduce_type(const at::Tensor& x, int op) {
  if (x.scalar_type() == at::kChar) return op == GS_SUM ? at::kInt : at::kChar;
  return x.scalar_type();
}

// reduce(x, n_access, op, scale, out_dtype, out)
PyObject* py_reduce(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 6, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const int64_t na = integer(p[1]);
    const int op = code(p[2]);
    const double scale = PyFloat_AsDouble(p[3]);
    if (scale == -1.0 && PyErr_Occurred()) throw Failed{};
    const auto sizes = x.sizes();
    // a leading slice as Python takes it: a negative end counts from the back
    const int64_t dims = x.dim(), lead = na < 0 ? (na + dims > 0 ? na + dims : 0) : na < dims ? na : dims;
    Result out(p[5], p[4], reduce_type(x, op), sizes.data(), int(lead), x);
    r = out.object;
    gs_ap xa = describe(x, 0), oa = describe_all(out.value);
    xa.n_access = int32_t(na);
    void* s = stream_of(x);
    call("reduce", [&] { return api.reduce(&xa, op, float(scale), &oa, s); });
  });
}

// windows_reduce(x, n_access, window, stride, pad_lo, pad_hi, op, scale, out_dtype, out)
PyObject* py_windows_reduce(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 10, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const int64_t na = integer(p[1]);
    const Ints window(p[2]), stride(p[3]), lo(p[4]), hi(p[5]);
    const int op = code(p[6]);
    const double scale = PyFloat_AsDouble(p[7]);
    if (scale == -1.0 && PyErr_Occurred()) throw Failed{};
    gs_ap xa = describe(x, 0), want{};
    xa.n_access = int32_t(na);
    if (p[9] == Py_None)
      call("windows_out_shape", [&] { return api.windows_out_shape(&xa, window.get(), stride.get(), lo.get(), hi.get(), &want); });
    Result out(p[9], p[8], reduce_type(x, op), want.shape, want.n_access, x);
    r = out.object;
    gs_ap oa = describe_all(out.value);
    void* s = stream_of(x);
    call("windows_reduce", [&] {
      return api.windows_reduce(&xa, window.get(), stride.get(), lo.get(), hi.get(), op, float(scale), &oa, s);
    });
  });
}

// access_windows(x, n_access, window, stride, pad_lo, pad_hi, pad_mode, out)
PyObject* py_access_windows(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 8, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const int64_t na = integer(p[1]);
    const Ints window(p[2]), stride(p[3]), lo(p[4]), hi(p[5]);
    const int mode = code(p[6]);
    gs_ap xa = describe(x, 0), want{};
    xa.n_access = int32_t(na);
    call("windows_out_shape", [&] { return api.windows_out_shape(&xa, window.get(), stride.get(), lo.get(), hi.get(), &want); });
    Result out(p[7], Py_None, x.scalar_type(), want.shape, want.rank, x);
    r = out.object;
    gs_ap oa = describe(out.value, na + window.n);
    void* s = stream_of(x);
    call("access_windows", [&] {
      return api.access_windows(&xa, window.get(), stride.get(), lo.get(), hi.get(), mode, &oa, s);
    });
  });
}

// depthwise_conv2d(x, w, stride, pad, act, out_dtype, out)
PyObject* py_depthwise(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 7, [&](PyObject*& r) {
    const at::Tensor &x = tensor(p[0]), &w = tensor(p[1]);
    const Ints stride(p[2]), pad(p[3]);
    const int act = code(p[4]);
    gs_ap xa = describe(x, 1), wa = describe(w, 1), want{};
    if (p[6] == Py_None) {
      if (w.dim() < 3) {
        PyErr_SetString(PyExc_IndexError, "weights (C,Kh,Kw) are wanted");
        throw Failed{};
      }
      const int64_t window[2] = {w.size(1), w.size(2)};
      gs_ap planes = xa;
      planes.n_access = 2;
      call("windows_out_shape", [&] { return api.windows_out_shape(&planes, window, stride.get(), pad.get(), pad.get(), &want); });
    }
    Result out(p[6], p[5], sum_type(x), want.shape, 4, x);
    r = out.object;
    gs_ap oa = describe(out.value, 4);
    void* s = stream_of(x);
    call("depthwise_conv2d", [&] { return api.depthwise_conv2d(&xa, &wa, stride.get(), pad.get(), act, &oa, s); });
  });
}

// pair_reduce(a, b, op, act, out)
PyObject* py_pair_reduce(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 5, [&](PyObject*& r) {
    const at::Tensor &a = tensor(p[0]), &b = tensor(p[1]);
    const int op = code(p[2]), act = code(p[3]);
    Result out(p[4], Py_None, a.scalar_type(), a.sizes().data(), int(a.dim()), a);
    r = out.object;
    gs_ap xa = describe_all(a), ya = describe_all(b), oa = describe_all(out.value);
    void* s = stream_of(a);
    call("pair_reduce", [&] { return api.pair_reduce(&xa, &ya, op, act, &oa, s); });
  });
}

// transpose(x, n_access, perm, out)
PyObject* py_transpose(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 4, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const int64_t na = integer(p[1]);
    const Ints perm(p[2]);
    int64_t shape[2 * GS_MAX_RANK];
    if (p[3] == Py_None)
      for (int i = 0; i < perm.n; ++i) {
        const int64_t d = perm.v[i] < 0 ? perm.v[i] + x.dim() : perm.v[i];
        if (d < 0 || d >= x.dim()) {
          PyErr_SetString(PyExc_IndexError, "tuple index out of range");
          throw Failed{};
        }
        shape[i] = x.size(d);
      }
    Result out(p[3], Py_None, x.scalar_type(), shape, perm.n, x);
    r = out.object;
    gs_ap xa = describe(x, 0), oa = describe(out.value, 0);
    xa.n_access = oa.n_access = int32_t(na);
    void* s = stream_of(x);
    call("transpose", [&] { return api.transpose(&xa, perm.get(), &oa, s); });
  });
}

// program_eval(text, tensors by name, integers by name, out_dtype, out, workspace)
PyObject* py_program_eval(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 6, [&](PyObject*& r) {
    const char* text = PyUnicode_AsUTF8(p[0]);
    if (!text) throw Failed{};
    // Names and tensors are held: the caller's mappings may change meanwhile, from another thread while the
    // interpreter lock is released, or from the conversion of an integer.
    const Items named(p[1]), numbers(p[2]);
    auto name_of = [](PyObject* key) {
      const char* s = PyUnicode_AsUTF8(key);
      if (!s) throw Failed{};
      return s;
    };
    std::vector<gs_named_ap> tensors;
    std::vector<gs_named_int> ints;
    const at::Tensor* first = nullptr;
    for (const auto& [key, value] : named.items) {
      const at::Tensor& t = tensor(value);
      if (!first) first = &t;
      tensors.push_back({name_of(key), describe(t, 0)});
    }
    for (const auto& [key, value] : numbers.items) ints.push_back({name_of(key), integer(value)});
    if (!first) {
      PyErr_SetString(PyExc_StopIteration, "a program needs a tensor");
      throw Failed{};
    }
    const int nt = int(tensors.size()), ni = int(ints.size());
    gs_ap want{};
    call("program_shape", [&] { return api.program_shape(text, tensors.data(), nt, ints.data(), ni, &want); });
    constexpr at::ScalarType types[5] = {at::kChar, at::kInt, at::kBFloat16, at::kFloat, at::kFloat8_e4m3fn};   // by gs_dtype
    Result out(p[4], p[3], types[want.dtype], want.shape, want.rank, *first);
    r = out.object;
    at::Tensor ws;
    if (p[5] != Py_None) {
      ws = tensor(p[5]);
    } else {
      const size_t need = api.program_workspace(text, tensors.data(), nt, ints.data(), ni);
      ws = at::empty({int64_t(need > 16 ? need : 16)}, at::TensorOptions().dtype(at::kByte).device(first->device()));
    }
    // the result as the program's access pattern, whatever shape its tensor has: as many elements, at least
    gs_ap oa = describe(out.value, 0);
    int64_t elements = 1;
    for (int i = 0; i < want.rank; ++i) elements *= want.shape[i];
    if (out.value.numel() < elements) refuse(GS_ERR_SHAPE, "program_eval");
    oa.rank = want.rank;
    oa.n_access = want.n_access;
    for (int i = 0; i < want.rank; ++i) oa.shape[i] = want.shape[i];
    void *wsp = ws.data_ptr(), *s = stream_of(*first);
    const size_t bytes = size_t(ws.numel());
    call("program_eval", [&] { return api.program_eval(text, tensors.data(), nt, ints.data(), ni, &oa, wsp, bytes, s); });
  });
}

// ---------------------------------------------------------------------------------------------
// microscaled 4-bit floats
// ---------------------------------------------------------------------------------------------

// Storage of one byte per element, dense.
void* bytes_of(const at::Tensor& t) {
  if (t.element_size() != 1 || !t.is_contiguous()) {
    PyErr_SetString(PyExc_ValueError, "4-bit and 8-bit numbers, scales of 4-bit ones, caches and workspaces are dense tensors of bytes");
    throw Failed{};
  }
  return t.data_ptr();
}

// All operands of a call lie on one device.
void same_device(const at::Tensor& a, std::initializer_list<const at::Tensor*> others) {
  for (const at::Tensor* t : others)
    if (t->defined() && t->device() != a.device()) {
      PyErr_SetString(PyExc_ValueError, "the tensors of a call are on one device");
      throw Failed{};
    }
}

PyObject* item(PyObject* tuple, Py_ssize_t i, Py_ssize_t size, const char* what) {
  if (!PyTuple_Check(tuple) || PyTuple_GET_SIZE(tuple) != size) {
    PyErr_Format(PyExc_TypeError, "%s is wanted", what);
    throw Failed{};
  }
  return PyTuple_GET_ITEM(tuple, i);
}

// binding.Mx4: (values, scales, shape, n_access)
struct Mx4 {
  at::Tensor values, scales;
  gs_mx4 d{};
  explicit Mx4(PyObject* o) : values(tensor(item(o, 0, 4, "an Mx4"))), scales(tensor(item(o, 1, 4, "an Mx4"))) {
    d.values = bytes_of(values);
    d.scales = bytes_of(scales);
    const Ints shape(item(o, 2, 4, "an Mx4"));
    pattern(shape.v, shape.n, integer(item(o, 3, 4, "an Mx4")));
    size_t need_values = 0, need_scales = 0;
    call("mx4_sizes", [&] { return api.mx4_sizes(&d, &need_values, &need_scales); });
    if (size_t(values.numel()) < need_values || size_t(scales.numel()) < need_scales) refuse(GS_ERR_SHAPE, "Mx4");
    same_device(values, {&scales});
  }
  // New storage for a pattern.
  Mx4(const int64_t* shape, int64_t rank, int64_t n_access, const at::Tensor& like) {
    pattern(shape, rank, n_access);
    size_t need_values = 0, need_scales = 0;
    call("mx4_sizes", [&] { return api.mx4_sizes(&d, &need_values, &need_scales); });
    int64_t rows = 1, v[GS_MAX_RANK + 2];
    for (int64_t i = 0; i < n_access; ++i) rows *= v[i] = shape[i];
    const auto bytes = at::TensorOptions().dtype(at::kByte).device(like.device());
    const int64_t pitch = rows ? int64_t(need_scales) / rows : 0, blocks = rows ? int64_t(need_values) / rows / 16 : 0;
    v[n_access] = pitch;
    scales = at::empty(at::IntArrayRef(v, size_t(n_access) + 1), bytes);
    v[n_access] = blocks;
    v[n_access + 1] = 16;
    values = at::empty(at::IntArrayRef(v, size_t(n_access) + 2), bytes);
    d.values = values.data_ptr();
    d.scales = scales.data_ptr();
  }

 private:
  void pattern(const int64_t* shape, int64_t rank, int64_t n_access) {
    if (rank > GS_MAX_RANK) {
      PyErr_SetString(PyExc_ValueError, "rank above GS_MAX_RANK");
      throw Failed{};
    }
    if (n_access < 0 || n_access > rank) refuse(GS_ERR_RANK, "Mx4");
    d.rank = int32_t(rank);
    d.n_access = int32_t(n_access);
    for (int64_t i = 0; i < rank; ++i) d.shape[i] = shape[i];
  }
};

// binding.Mx4Cache: (data, page_size, head_dim), data (pages, heads, bytes of a block)
struct Cache {
  at::Tensor data;
  gs_mx4_cache d{};
  explicit Cache(PyObject* o) : data(tensor(item(o, 0, 3, "an Mx4Cache"))) {
    d.data = bytes_of(data);
    const int64_t page = integer(item(o, 1, 3, "an Mx4Cache")), dim = integer(item(o, 2, 3, "an Mx4Cache"));
    if (data.dim() != 3 || data.size(1) > INT32_MAX || page < 0 || page > INT32_MAX || dim < 0 || dim > INT32_MAX) refuse(GS_ERR_SHAPE, "Mx4Cache");
    d.n_pages = data.size(0);
    d.heads = int32_t(data.size(1));
    d.page_size = int32_t(page);
    d.head_dim = int32_t(dim);
    // (where the description is impossible, the entry point says why)
    const size_t need = api.mx4_cache_bytes(&d);
    if (need && size_t(data.numel()) != need) refuse(GS_ERR_SHAPE, "Mx4Cache");
  }
};

at::Tensor workspace_for(PyObject* given, size_t need, const at::Tensor& like) {
  if (given != Py_None) {
    const at::Tensor ws = tensor(given);
    bytes_of(ws);
    return ws;
  }
  return need ? at::empty({int64_t(need)}, at::TensorOptions().dtype(at::kByte).device(like.device())) : at::Tensor();
}

// mx4_quantize(x, n_access, out) -> (values, scales); out: an Mx4 or None
PyObject* py_mx4_quantize(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 3, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const gs_ap xa = describe(x, integer(p[1]));
    Mx4 out = p[2] == Py_None ? Mx4(xa.shape, xa.rank, xa.n_access, x) : Mx4(p[2]);
    same_device(x, {&out.values});
    void* s = stream_of(x);
    call("mx4_quantize", [&] { return api.mx4_quantize(&xa, &out.d, s); });
    const Owned values(THPVariable_Wrap(out.values)), scales(THPVariable_Wrap(out.scales));
    r = PyTuple_Pack(2, values.object, scales.object);
    if (!r) throw Failed{};
  });
}

// mx4_dequantize(m, out_dtype, out)
PyObject* py_mx4_dequantize(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 3, [&](PyObject*& r) {
    const Mx4 m(p[0]);
    Result out(p[2], p[1], at::kBFloat16, m.d.shape, m.d.rank, m.values);
    r = out.object;
    gs_ap oa = describe(out.value, m.d.n_access);
    same_device(m.values, {&out.value});
    void* s = stream_of(m.values);
    call("mx4_dequantize", [&] { return api.mx4_dequantize(&m.d, &oa, s); });
  });
}

// mx4_dot(a0, a1, out_dtype, act, out, workspace)
PyObject* py_mx4_dot(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 6, [&](PyObject*& r) {
    const Mx4 a0(p[0]), a1(p[1]);
    const int act = code(p[3]);
    int64_t shape[2 * GS_MAX_RANK];
    int rank = 0;
    for (int i = 0; i < a0.d.n_access; ++i) shape[rank++] = a0.d.shape[i];
    for (int i = 0; i < a1.d.n_access; ++i) shape[rank++] = a1.d.shape[i];
    Result out(p[4], p[2], at::kFloat, shape, rank, a0.values);
    r = out.object;
    gs_ap oa = describe_all(out.value);
    const at::Tensor ws = workspace_for(p[5], api.mx4_dot_workspace(&a0.d, &a1.d), a0.values);
    same_device(a0.values, {&a1.values, &out.value, &ws});
    void *s = stream_of(a0.values), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? size_t(ws.numel()) : 0;
    call("mx4_dot", [&] { return api.mx4_dot(&a0.d, &a1.d, &oa, act, w, bytes, s); });
  });
}

// mx4_weight_dot(x, w, n_access, out_dtype, act, out, workspace)
PyObject* py_mx4_weight_dot(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 7, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const Mx4 a1(p[1]);
    const gs_ap xa = describe(x, integer(p[2]));
    const int act = code(p[4]);
    int64_t shape[2 * GS_MAX_RANK];
    int rank = 0;
    for (int i = 0; i < xa.n_access && i < xa.rank; ++i) shape[rank++] = xa.shape[i];
    for (int i = 0; i < a1.d.n_access; ++i) shape[rank++] = a1.d.shape[i];
    Result out(p[5], p[3], at::kFloat, shape, rank, x);
    r = out.object;
    gs_ap oa = describe_all(out.value);
    const at::Tensor ws = workspace_for(p[6], api.mx4_weight_dot_workspace(&xa, &a1.d), x);
    same_device(x, {&a1.values, &out.value, &ws});
    void *s = stream_of(x), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? size_t(ws.numel()) : 0;
    call("mx4_weight_dot", [&] { return api.mx4_weight_dot(&xa, &a1.d, &oa, act, w, bytes, s); });
  });
}

// mx4_cache_append(cache, table, first, counts, k, v)
PyObject* py_mx4_cache_append(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 6, [&](PyObject*& r) {
    const Cache cache(p[0]);
    const at::Tensor &table = tensor(p[1]), &first = tensor(p[2]), &k = tensor(p[4]), &v = tensor(p[5]);
    const at::Tensor counts = p[3] == Py_None ? at::Tensor() : tensor(p[3]);
    same_device(cache.data, {&table, &first, &counts, &k, &v});
    const gs_ap ta = describe(table, 1), fa = describe(first, 1), ka = describe(k, 3), va = describe(v, 3);
    gs_ap ca{};
    if (counts.defined()) ca = describe(counts, 1);
    void* s = stream_of(cache.data);
    call("mx4_cache_append", [&] { return api.mx4_cache_append(&cache.d, &ta, &fa, counts.defined() ? &ca : nullptr, &ka, &va, s); });
    Py_INCREF(Py_None);
    r = Py_None;
  });
}

// mx4_cache_read(cache, table, first, n_tokens, out_dtype, k, v) -> (k, v)
PyObject* py_mx4_cache_read(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 7, [&](PyObject*& r) {
    const Cache cache(p[0]);
    const at::Tensor &table = tensor(p[1]), &first = tensor(p[2]);
    const int64_t tokens = integer(p[3]);
    if (tokens < 0 || table.dim() < 1) refuse(GS_ERR_SHAPE, "mx4_cache_read");
    const int64_t shape[4] = {table.size(0), tokens, cache.d.heads, cache.d.head_dim};
    const Result k(p[5], p[4], at::kBFloat16, shape, 4, cache.data);
    const Owned k_held(k.object);
    const Result v(p[6], p[4], at::kBFloat16, shape, 4, cache.data);
    const Owned v_held(v.object);
    same_device(cache.data, {&table, &first, &k.value, &v.value});
    const gs_ap ta = describe(table, 1), fa = describe(first, 1);
    gs_ap ka = describe(k.value, 3), va = describe(v.value, 3);
    if (k.value.dim() > 1 && k.value.size(1) != tokens) refuse(GS_ERR_SHAPE, "mx4_cache_read");
    void* s = stream_of(cache.data);
    call("mx4_cache_read", [&] { return api.mx4_cache_read(&cache.d, &ta, &fa, &ka, &va, s); });
    r = PyTuple_Pack(2, k.object, v.object);
    if (!r) throw Failed{};
  });
}

// mx4_attend(q, cache, table, lengths, scale, window, sinks, out_dtype, out, workspace)
PyObject* py_mx4_attend(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 10, [&](PyObject*& r) {
    const at::Tensor &q = tensor(p[0]), &table = tensor(p[2]), &lengths = tensor(p[3]);
    const Cache cache(p[1]);
    const double scale = PyFloat_AsDouble(p[4]);
    if (scale == -1.0 && PyErr_Occurred()) throw Failed{};
    const int64_t window = integer(p[5]), sinks = integer(p[6]);
    const gs_ap qa = describe(q, 3), ta = describe(table, 1), la = describe(lengths, 1);
    Result out(p[8], p[7], at::kBFloat16, qa.shape, qa.rank, q);
    r = out.object;
    gs_ap oa = describe(out.value, 3);
    const at::Tensor ws = workspace_for(p[9], p[9] == Py_None ? api.mx4_attend_workspace(&qa, &cache.d, &ta) : 0, q);
    same_device(q, {&cache.data, &table, &lengths, &out.value, &ws});
    void *s = stream_of(q), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? size_t(ws.numel()) : 0;
    call("mx4_attend", [&] { return api.mx4_attend(&qa, &cache.d, &ta, &la, float(scale), window, sinks, &oa, w, bytes, s); });
  });
}

// New tensors that are made and dropped together, in one allocation: each costs the caller a microsecond.
struct Together {
  at::Tensor bytes;
  size_t used = 0;
  Together(size_t total, const at::Tensor& like) : bytes(at::empty({int64_t(total)}, at::TensorOptions().dtype(at::kByte).device(like.device()))) {}
  static size_t room(size_t n) { return (n + 511) / 512 * 512; }      // (as aligned as allocations are)
  at::Tensor take(at::IntArrayRef sizes, at::ScalarType type) {
    const size_t item = c10::elementSize(type);
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(bytes.storage()), bytes.key_set(), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_storage_offset(int64_t(used / item));
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    used += room(size_t(t.numel()) * item);
    return t;
  }
};

// binding.F8: (values, scales, shape, n_access, block_rows)
struct F8 {
  at::Tensor values, scales;
  gs_f8 d{};
  explicit F8(PyObject* o) : values(tensor(item(o, 0, 5, "an F8"))), scales(tensor(item(o, 1, 5, "an F8"))) {
    d.values = bytes_of(values);
    if (scales.scalar_type() != at::kFloat || !scales.is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "scales are dense tensors of float32");
      throw Failed{};
    }
    d.scales = scales.data_ptr();
    const Ints shape(item(o, 2, 5, "an F8"));
    pattern(shape.v, shape.n, integer(item(o, 3, 5, "an F8")), integer(item(o, 4, 5, "an F8")));
    sizes();
    if (size_t(values.numel()) < need_values || size_t(scales.numel()) * 4 < need_scales) refuse(GS_ERR_SHAPE, "F8");
    same_device(values, {&scales});
  }
  // New storage for a pattern.
  F8(const int64_t* shape, int64_t rank, int64_t n_access, int64_t block_rows, const at::Tensor& like) {
    pattern(shape, rank, n_access, block_rows);
    sizes();
    int64_t cols = 1, v[GS_MAX_RANK + 2];
    for (int64_t i = n_access; i < rank; ++i) cols *= shape[i];
    for (int64_t i = 0; i < n_access; ++i) v[i] = shape[i];
    v[n_access] = (cols + 127) / 128;
    v[n_access + 1] = 128;
    Together both(Together::room(need_values) + need_scales, like);
    values = both.take(at::IntArrayRef(v, size_t(n_access) + 2), at::kFloat8_e4m3fn);
    if (n_access > 0) v[n_access - 1] = (v[n_access - 1] + block_rows - 1) / block_rows;
    v[n_access] = (v[n_access] + 3) / 4 * 4;
    scales = both.take(at::IntArrayRef(v, size_t(n_access) + 1), at::kFloat);
    d.values = values.data_ptr();
    d.scales = scales.data_ptr();
  }

 private:
  size_t need_values = 0, need_scales = 0;
  void sizes() {
    const int status = api.f8_sizes(&d, &need_values, &need_scales);
    if (status != GS_OK) refuse(status, "F8");
  }
  void pattern(const int64_t* shape, int64_t rank, int64_t n_access, int64_t block_rows) {
    if (rank > GS_MAX_RANK) {
      PyErr_SetString(PyExc_ValueError, "rank above GS_MAX_RANK");
      throw Failed{};
    }
    if (n_access < 0 || n_access > rank) refuse(GS_ERR_RANK, "F8");
    if (block_rows != 1 && block_rows != 128) refuse(GS_ERR_UNSUPPORTED, "F8");
    d.rank = int32_t(rank);
    d.n_access = int32_t(n_access);
    d.block_rows = int32_t(block_rows);
    for (int64_t i = 0; i < rank; ++i) d.shape[i] = shape[i];
  }
};

at::Tensor optional_tensor(PyObject* o) { return o == Py_None ? at::Tensor() : tensor(o); }

// f8_quantize(x, n_access, block_rows, out) -> (values, scales); out: an F8 or None
PyObject* py_f8_quantize(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 4, [&](PyObject*& r) {
    const at::Tensor& x = tensor(p[0]);
    const gs_ap xa = describe(x, integer(p[1]));
    F8 out = p[3] == Py_None ? F8(xa.shape, xa.rank, xa.n_access, integer(p[2]), x) : F8(p[3]);
    same_device(x, {&out.values});
    void* s = stream_of(x);
    call("f8_quantize", [&] { return api.f8_quantize(&xa, &out.d, s); });
    const Owned values(THPVariable_Wrap(out.values)), scales(THPVariable_Wrap(out.scales));
    r = PyTuple_Pack(2, values.object, scales.object);
    if (!r) throw Failed{};
  });
}

// f8_dequantize(m, out_dtype, out)
PyObject* py_f8_dequantize(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 3, [&](PyObject*& r) {
    const F8 m(p[0]);
    Result out(p[2], p[1], at::kBFloat16, m.d.shape, m.d.rank, m.values);
    r = out.object;
    gs_ap oa = describe(out.value, m.d.n_access);
    same_device(m.values, {&out.value});
    void* s = stream_of(m.values);
    call("f8_dequantize", [&] { return api.f8_dequantize(&m.d, &oa, s); });
  });
}

// norm(f8, x, weight, residual, eps, n_access, out_dtype, out, sum) -> f8: (values, scales, sum), else (out, sum); sum is
// x itself where there is no residual and no tensor for it is given
PyObject* py_norm(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 9, [&](PyObject*& r) {
    const bool f8 = p[0] == Py_True;
    const at::Tensor& x = tensor(p[1]);
    const at::Tensor weight = optional_tensor(p[2]), residual = optional_tensor(p[3]);
    const double eps = PyFloat_AsDouble(p[4]);
    if (eps == -1.0 && PyErr_Occurred()) throw Failed{};
    const gs_ap xa = describe(x, integer(p[5]));
    gs_ap wa{}, ra{}, sa{};
    if (weight.defined()) wa = describe(weight, 0);
    if (residual.defined()) ra = describe(residual, xa.n_access);
    at::Tensor sum;
    if (p[8] != Py_None) sum = tensor(p[8]);
    else if (residual.defined()) sum = at::empty(x.sizes(), x.options());
    if (sum.defined()) sa = describe(sum, xa.n_access);
    same_device(x, {&weight, &residual, &sum});
    void* s = stream_of(x);
    const gs_ap *w = weight.defined() ? &wa : nullptr, *res = residual.defined() ? &ra : nullptr;
    gs_ap* total = sum.defined() ? &sa : nullptr;
    const Owned total_held(THPVariable_Wrap(sum.defined() ? sum : x));
    if (f8) {
      F8 out = p[7] == Py_None ? F8(xa.shape, xa.rank, xa.n_access, 1, x) : F8(p[7]);
      same_device(x, {&out.values});
      call("f8_norm", [&] { return api.f8_norm(&xa, res, w, float(eps), total, &out.d, s); });
      const Owned values(THPVariable_Wrap(out.values)), scales(THPVariable_Wrap(out.scales));
      r = PyTuple_Pack(3, values.object, scales.object, total_held.object);
    } else {
      const Result out(p[7], p[6], x.scalar_type(), xa.shape, xa.rank, x);
      const Owned out_held(out.object);
      same_device(x, {&out.value});
      gs_ap oa = describe(out.value, xa.n_access);
      call("norm", [&] { return api.norm(&xa, res, w, float(eps), total, &oa, s); });
      r = PyTuple_Pack(2, out.object, total_held.object);
    }
    if (!r) throw Failed{};
  });
}

// f8_dot(a0, a1, out_dtype, act, out, workspace)
PyObject* py_f8_dot(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 6, [&](PyObject*& r) {
    const F8 a0(p[0]), a1(p[1]);
    const int act = code(p[3]);
    int64_t shape[2 * GS_MAX_RANK];
    int rank = 0;
    for (int i = 0; i < a0.d.n_access; ++i) shape[rank++] = a0.d.shape[i];
    for (int i = 0; i < a1.d.n_access; ++i) shape[rank++] = a1.d.shape[i];
    Result out(p[4], p[2], at::kFloat, shape, rank, a0.values);
    r = out.object;
    gs_ap oa = describe_all(out.value);
    const at::Tensor ws = workspace_for(p[5], p[5] == Py_None ? api.f8_dot_workspace(&a0.d, &a1.d) : 0, a0.values);
    same_device(a0.values, {&a1.values, &out.value, &ws});
    void *s = stream_of(a0.values), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? size_t(ws.numel()) : 0;
    call("f8_dot", [&] { return api.f8_dot(&a0.d, &a1.d, &oa, act, w, bytes, s); });
  });
}

// f8_expert_dot(a0, w, offsets, tokens, out_dtype, act, out, workspace)
PyObject* py_f8_expert_dot(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 8, [&](PyObject*& r) {
    const F8 a0(p[0]), a1(p[1]);
    const at::Tensor& offsets = tensor(p[2]);
    const at::Tensor tokens = optional_tensor(p[3]);
    const int act = code(p[5]);
    if (tokens.defined() && tokens.dim() != 1) refuse(GS_ERR_RANK, "f8_expert_dot");
    int64_t shape[2] = {1, a1.d.n_access > 0 ? a1.d.shape[a1.d.n_access - 1] : 1};
    if (tokens.defined()) shape[0] = tokens.size(0);
    else
      for (int i = 0; i < a0.d.n_access; ++i) shape[0] *= a0.d.shape[i];
    Result out(p[6], p[4], at::kFloat, shape, 2, a0.values, true);
    r = out.object;
    const gs_ap fa = describe(offsets, 1);
    gs_ap ta{}, oa = describe_all(out.value);
    if (tokens.defined()) ta = describe(tokens, 1);
    const at::Tensor ws = workspace_for(p[7], p[7] == Py_None ? api.f8_expert_dot_workspace(&a0.d, shape[0], &a1.d) : 0, a0.values);
    same_device(a0.values, {&a1.values, &offsets, &tokens, &out.value, &ws});
    void *s = stream_of(a0.values), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? size_t(ws.numel()) : 0;
    call("f8_expert_dot", [&] { return api.f8_expert_dot(&a0.d, tokens.defined() ? &ta : nullptr, &fa, &a1.d, &oa, act, w, bytes, s); });
  });
}

// expert_sort(experts, n_experts, out, workspace) -> (offsets, tokens, places); out: three tensors or None
PyObject* py_expert_sort(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 4, [&](PyObject*& r) {
    const at::Tensor& experts = tensor(p[0]);
    const int64_t n_experts = integer(p[1]);
    if (n_experts < 0) refuse(GS_ERR_SHAPE, "expert_sort");
    if (n_experts > 4096) refuse(GS_ERR_UNSUPPORTED, "expert_sort");    // (before offsets for them are made)
    at::Tensor offsets, tokens, places;
    if (p[2] != Py_None) {
      offsets = tensor(item(p[2], 0, 3, "an ExpertSort"));
      tokens = tensor(item(p[2], 1, 3, "an ExpertSort"));
      places = tensor(item(p[2], 2, 3, "an ExpertSort"));
      if (offsets.dim() == 1 && offsets.size(0) != n_experts + 1) refuse(GS_ERR_SHAPE, "expert_sort");
    } else {
      const size_t all = size_t(experts.numel()) * 4;
      Together three(Together::room(size_t(n_experts + 1) * 4) + Together::room(all) + all, experts);
      offsets = three.take({n_experts + 1}, at::kInt);
      tokens = three.take({experts.numel()}, at::kInt);
      places = three.take(experts.sizes(), at::kInt);
    }
    const gs_ap ea = describe_all(experts);
    gs_ap oa = describe_all(offsets), ta = describe_all(tokens), pa = describe_all(places);
    const at::Tensor ws = workspace_for(p[3], p[3] == Py_None ? api.expert_sort_workspace(experts.numel(), n_experts) : 0, experts);
    same_device(experts, {&offsets, &tokens, &places, &ws});
    void *s = stream_of(experts), *w = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t bytes = ws.defined() ? size_t(ws.numel()) : 0;
    call("expert_sort", [&] { return api.expert_sort(&ea, &oa, &ta, &pa, w, bytes, s); });
    const Owned o(THPVariable_Wrap(offsets)), t(THPVariable_Wrap(tokens)), q(THPVariable_Wrap(places));
    r = PyTuple_Pack(3, o.object, t.object, q.object);
    if (!r) throw Failed{};
  });
}

// A shape like `of`'s with another first dimension.
struct RowsShape {
  int64_t v[GS_MAX_RANK];
  int rank;
  RowsShape(const at::Tensor& of, int64_t first) : rank(int(of.dim())) {
    if (rank < 1 || rank > GS_MAX_RANK) {
      PyErr_SetString(PyExc_ValueError, "tokens and rows have 1 to 8 dimensions");
      throw Failed{};
    }
    for (int i = 0; i < rank; ++i) v[i] = i ? of.size(i) : first;
  }
};

// expert_split(x, places, out)
PyObject* py_expert_split(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 3, [&](PyObject*& r) {
    const at::Tensor &x = tensor(p[0]), &places = tensor(p[1]);
    const RowsShape shape(x, places.numel());
    Result rows(p[2], Py_None, x.scalar_type(), shape.v, shape.rank, x, true);
    r = rows.object;
    const gs_ap xa = describe(x, 1), pa = describe_all(places);
    gs_ap ra = describe(rows.value, 1);
    same_device(x, {&places, &rows.value});
    void* s = stream_of(x);
    call("expert_split", [&] { return api.expert_split(&xa, &pa, &ra, s); });
  });
}

// expert_join(rows, places, weights, out_dtype, out)
PyObject* py_expert_join(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 5, [&](PyObject*& r) {
    const at::Tensor &rows = tensor(p[0]), &places = tensor(p[1]);
    const at::Tensor weights = optional_tensor(p[2]);
    const RowsShape shape(rows, places.dim() ? places.size(0) : 0);
    Result out(p[4], p[3], rows.scalar_type(), shape.v, shape.rank, rows);
    r = out.object;
    const gs_ap ra = describe(rows, 1), pa = describe_all(places);
    gs_ap wa{}, oa = describe(out.value, 1);
    if (weights.defined()) wa = describe_all(weights);
    same_device(rows, {&places, &weights, &out.value});
    void* s = stream_of(rows);
    call("expert_join", [&] { return api.expert_join(&ra, &pa, weights.defined() ? &wa : nullptr, &oa, s); });
  });
}

// expert_join_grad(grad, rows, places, weights, grad_rows, grad_weights) -> (grad_rows, grad_weights)
PyObject* py_expert_join_grad(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 6, [&](PyObject*& r) {
    const at::Tensor &grad = tensor(p[0]), &rows = tensor(p[1]), &places = tensor(p[2]);
    const at::Tensor weights = optional_tensor(p[3]);
    const RowsShape shape(rows, rows.dim() ? rows.size(0) : 0);
    const Result grad_rows(p[4], Py_None, rows.scalar_type(), shape.v, shape.rank, rows, true);
    const Owned rows_held(grad_rows.object);
    const Result grad_weights(p[5], Py_None, at::kFloat, places.sizes().data(), int(places.dim()), rows);
    const Owned weights_held(grad_weights.object);
    const gs_ap ga = describe(grad, 1), ra = describe(rows, 1), pa = describe_all(places);
    gs_ap wa{}, gra = describe(grad_rows.value, 1), gwa = describe_all(grad_weights.value);
    if (weights.defined()) wa = describe_all(weights);
    same_device(grad, {&rows, &places, &weights, &grad_rows.value, &grad_weights.value});
    void* s = stream_of(grad);
    call("expert_join_grad", [&] { return api.expert_join_grad(&ga, &ra, &pa, weights.defined() ? &wa : nullptr, &gra, &gwa, s); });
    r = PyTuple_Pack(2, grad_rows.object, grad_weights.object);
    if (!r) throw Failed{};
  });
}

// bind(addresses by entry point name, GlensideError)
PyObject* py_bind(PyObject*, PyObject* const* p, Py_ssize_t n) {
  return guarded(n, 2, [&](PyObject*& r) {
    auto get = [&](const char* name, auto& fn) {
      PyObject* v = PyDict_GetItemString(p[0], name);
      if (!v) {
        PyErr_SetString(PyExc_KeyError, name);
        throw Failed{};
      }
      fn = reinterpret_cast<std::decay_t<decltype(fn)>>(PyLong_AsVoidPtr(v));
      if (!fn) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, name);
        throw Failed{};
      }
    };
    get("glenside_windows_out_shape", api.windows_out_shape);
    get("glenside_access_windows", api.access_windows);
    get("glenside_cartesian_dot", api.cartesian_dot);
    get("glenside_conv2d_direct", api.conv2d_direct);
    get("glenside_conv2d_im2col", api.conv2d_im2col);
    get("glenside_conv2d_direct_packed", api.conv2d_direct_packed);
    get("glenside_conv2d_direct_packed_with_projection", api.conv2d_direct_packed_with_projection);
    get("glenside_conv2d_direct_workspace", api.conv2d_direct_workspace);
    get("glenside_conv2d_im2col_workspace", api.conv2d_im2col_workspace);
    get("glenside_reduce", api.reduce);
    get("glenside_windows_reduce", api.windows_reduce);
    get("glenside_pair_reduce", api.pair_reduce);
    get("glenside_depthwise_conv2d", api.depthwise_conv2d);
    get("glenside_transpose", api.transpose);
    get("glenside_program_shape", api.program_shape);
    get("glenside_program_workspace", api.program_workspace);
    get("glenside_program_eval", api.program_eval);
    get("glenside_mx4_sizes", api.mx4_sizes);
    get("glenside_mx4_quantize", api.mx4_quantize);
    get("glenside_mx4_dequantize", api.mx4_dequantize);
    get("glenside_mx4_dot", api.mx4_dot);
    get("glenside_mx4_dot_workspace", api.mx4_dot_workspace);
    get("glenside_mx4_weight_dot", api.mx4_weight_dot);
    get("glenside_mx4_weight_dot_workspace", api.mx4_weight_dot_workspace);
    get("glenside_mx4_cache_bytes", api.mx4_cache_bytes);
    get("glenside_mx4_cache_append", api.mx4_cache_append);
    get("glenside_mx4_cache_read", api.mx4_cache_read);
    get("glenside_mx4_attend", api.mx4_attend);
    get("glenside_mx4_attend_workspace", api.mx4_attend_workspace);
    get("glenside_f8_sizes", api.f8_sizes);
    get("glenside_f8_quantize", api.f8_quantize);
    get("glenside_f8_dequantize", api.f8_dequantize);
    get("glenside_norm", api.norm);
    get("glenside_f8_norm", api.f8_norm);
    get("glenside_f8_dot", api.f8_dot);
    get("glenside_f8_dot_workspace", api.f8_dot_workspace);
    get("glenside_f8_expert_dot", api.f8_expert_dot);
    get("glenside_f8_expert_dot_workspace", api.f8_expert_dot_workspace);
    get("glenside_expert_sort", api.expert_sort);
    get("glenside_expert_sort_workspace", api.expert_sort_workspace);
    get("glenside_expert_split", api.expert_split);
    get("glenside_expert_join", api.expert_join);
    get("glenside_expert_join_grad", api.expert_join_grad);
    Py_INCREF(p[1]);
    Py_XDECREF(error_class);
    error_class = p[1];
    Py_INCREF(Py_None);
    r = Py_None;
  });
}

#define GS_FN(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    GS_FN("bind", py_bind), GS_FN("cartesian_dot", py_cartesian_dot), GS_FN("conv", py_conv), GS_FN("conv_with_projection", py_conv_with_projection), GS_FN("reduce", py_reduce),
    GS_FN("windows_reduce", py_windows_reduce), GS_FN("access_windows", py_access_windows),
    GS_FN("depthwise_conv2d", py_depthwise), GS_FN("pair_reduce", py_pair_reduce), GS_FN("transpose", py_transpose),
    GS_FN("program_eval", py_program_eval),
    GS_FN("mx4_quantize", py_mx4_quantize), GS_FN("mx4_dequantize", py_mx4_dequantize), GS_FN("mx4_dot", py_mx4_dot),
    GS_FN("mx4_weight_dot", py_mx4_weight_dot), GS_FN("mx4_cache_append", py_mx4_cache_append),
    GS_FN("mx4_cache_read", py_mx4_cache_read), GS_FN("mx4_attend", py_mx4_attend),
    GS_FN("f8_quantize", py_f8_quantize), GS_FN("f8_dequantize", py_f8_dequantize), GS_FN("norm", py_norm), GS_FN("f8_dot", py_f8_dot),
    GS_FN("f8_expert_dot", py_f8_expert_dot), GS_FN("expert_sort", py_expert_sort), GS_FN("expert_split", py_expert_split),
    GS_FN("expert_join", py_expert_join), GS_FN("expert_join_grad", py_expert_join_grad),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
